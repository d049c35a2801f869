"""Scoring and losses of given tokens where sizes, options and values leave the ordinary, against 64 bits."""
import pytest

from tests import score_reference as ref
from tests.test_gpu_score import context, logits, out, preference, torch  # noqa: F401  (torch: a fixture)

pytestmark = pytest.mark.gpu


# The losses of up to 64 pairs are added up by one cluster of up to eight CTAs, which take the pairs in turn; of more, by a launch
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("pairs", [2, 7, 8, 9, 17, 64, 65, 200])
def test_preference_of_many_pairs(torch, pairs, dtype):  # noqa: F811
    """Short ragged sequences, a third of them empty; the loss of every pair, its rows' gradient, the total, the same bits every time."""
    dt, V = getattr(torch, dtype), 300
    lengths = torch.randint(0, 6, (2 * pairs,), generator=torch.Generator().manual_seed(pairs))
    lengths = torch.where(lengths < 2, 0, lengths)
    start = torch.cat([torch.zeros(1, dtype=torch.long), lengths.cumsum(0)]).int().cuda()
    n = max(1, int(start[-1]))
    z, tok, g = logits(torch, n, V, dt, pairs)
    tok[torch.rand(n, generator=g, device="cuda") < 0.2] = -1
    ctx = context(V, dt)
    pw = torch.rand(pairs, generator=g, device="cuda")
    for rule in ("sigmoid", "squared", "hinge"):
        preference(torch, ctx, z, z, tok, start, torch.full_like(z, 9.0), rule, pw=pw)
        preference(torch, ctx, z, z, tok, start, torch.full_like(z, 9.0), rule, average=True)
    want = None
    for _ in range(20):
        so, po, total = out(torch, 2 * pairs) + out(torch, pairs) + out(torch, 1)
        grad = torch.full_like(z, 9.0)
        scratch = torch.full((16 * n,), 255, dtype=torch.uint8, device="cuda")
        ctx.preference_loss(z, tok, start, po, so, scratch, pair_weight=pw, loss_out=total, grad_out=grad)
        assert float(total) == float(po.double().sum().float())          # (32-bit terms added in 64 bits: any order, one rounding)
        want = want or (so, po, total, grad)
        assert all(torch.equal(a, b) for a, b in zip((so, po, total, grad), want))
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype,V", [("bfloat16", 33538042), ("float32", 16769022)])
def test_rows_whose_last_segment_is_empty(torch, V, dtype):  # noqa: F811
    """A preference gradient cuts rows into segments of up to 2048 units by the units a row may have, one more than these rows
    have: 2048 segments, the last with none.  The last element, a segment's before it, is the token's."""
    dt = getattr(torch, dtype)
    N = 128 // torch.finfo(dt).bits
    assert (V + 2 * N - 2) // N == 2047 * 2048 + 1 and (V + N - 1) // N == (V + 2 + N - 1) // N == 2047 * 2048
    z, tok, _ = logits(torch, 2, V, dt, 5)
    tok[:] = V - 1
    ctx = context(V, dt)
    start = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    so, po = out(torch, 2)[0], out(torch, 1)[0]
    scratch = torch.empty(32, dtype=torch.uint8, device="cuda")
    grad = torch.full_like(z, 9.0)
    ctx.preference_loss(z, tok, start, po, so, scratch, rule="hinge", beta=0.01, grad_out=grad)
    assert 0.0 < float(po) < 2.0 and ctx.status() == 0      # (inside the hinge: dL/dl is -beta and beta)
    dl = torch.tensor([-0.01, 0.01], dtype=torch.float32, device="cuda").double()
    lnp, p, l, H, lse, on = ref.rows(z, tok)
    want, size = ref.gradient(lnp, p, H, tok, on, dl, 0 * dl, 1.0)
    # (a CTA folds 128 blocks of units into its sums, at most 10 roundings of 2^-24 each)
    ref.close_grad(grad, want, size, rel=ref.R + 1280 * 2.0 ** -24)
    assert grad[:, -1].tolist() == pytest.approx([-0.01, 0.01], rel=2.0 ** -8)
    ctx.preference_loss(z, tok, start, po, so, scratch, rule="hinge", beta=0.01, grad_out=z)
    assert torch.equal(z, grad)


def masked(torch, n, V, dt, seed, bias=0.0):
    """Logits with a third masked by -inf, some by the type's lowest value; tokens among what is left."""
    z, tok, g = logits(torch, n, V, dt, seed)
    z[::2] += bias
    z[:, 1::3] = float("-inf")
    z[:, 2::7] = torch.finfo(dt).min
    tok = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, z.argmax(-1).int(), (tok // 21) * 21)     # (21 k: a logit)
    return z, tok, g


LAUNCHES = [(3, 40), (3, 5000), (2, 140000), (400, 9001), (400, 20000), (300, 70000), (90, 151936), (700, 1000)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T", [1e-8, 1e-9, 1e-20, 1e-30])
@pytest.mark.parametrize("n,V", LAUNCHES)
def test_entropies_at_the_lowest_temperatures(torch, n, V, T, dtype):  # noqa: F811
    """Stretches of a row without a logit (masked, or behind a short row's end): nothing of them enters the entropy."""
    dt = getattr(torch, dtype)
    z, tok, g = masked(torch, n, V, dt, V)
    z[:, V // 8: 7 * V // 8] = float("-inf")
    tok = torch.where(z.gather(1, tok.long()[:, None])[:, 0] > -1e30, tok, 0)
    ctx = context(V, dt, T)
    T = float(torch.tensor(T, dtype=torch.float32))          # as the context holds it
    lnp, p, l, H, lse, on = ref.rows(z, tok, T)
    lp, ent, lo = out(torch, n, 3)
    ctx.token_logprob(z, tok, lp, ent, lo)
    ref.close_logp(lp, l)
    ref.close_logp(lo, lse)
    lnS = lse - z.double().amax(-1) / T
    ref.close_entropy(ent, H, torch.where(lnS.abs() < 20, lnS, 0.0))     # (lse of 1e9 and more holds no ln S: of size ln 2)
    grad = torch.full_like(z, 9.0)
    ctx.token_logprob_grad(z, tok, torch.ones(n, device="cuda"), grad, grad_entropy=torch.zeros(n, device="cuda"))
    want, size = ref.gradient(lnp, p, H, tok, on, torch.ones_like(l), torch.zeros_like(l), T)
    ref.close_grad(grad, want, size, rel=2 * ref.R)
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,dH", [(1e-3, 1.0), (1e-5, 1.0), (1e-9, 1.0), (1e-2, 65536.0), (1e-4, 1e6), (0.7, 1e12)])
@pytest.mark.parametrize("n,V", LAUNCHES)
def test_entropy_gradients_of_masked_logits(torch, n, V, T, dH, dtype):  # noqa: F811
    """Low temperatures and large coefficients: exponents of masked logits times a large factor stay finite, their gradient 0."""
    dt = getattr(torch, dtype)
    for bias in (0.0, 40.0):
        z, tok, g = masked(torch, n, V, dt, V, bias)
        ctx = context(V, dt, T)
        t = float(torch.tensor(T, dtype=torch.float32))      # as the context holds it
        a = torch.randn(n, generator=g, device="cuda")
        b = dH * torch.randn(n, generator=g, device="cuda")
        lnp, p, l, H, lse, on = ref.rows(z, tok, t)
        grad = torch.full_like(z, 9.0)
        ctx.token_logprob_grad(z, tok, a, grad, grad_entropy=b)
        assert ctx.status() == 0 and bool(torch.isfinite(grad).all())
        assert bool((grad[:, 1::3][z[:, 1::3] == float("-inf")] == 0).all()) and bool((grad[z <= -1e30] == 0).all())
        want, size = ref.gradient(lnp, p, H, tok, on, a.double(), b.double(), t)
        # H of the device enters as ln S - T / S, two numbers of the size of ln V that cancel: 2 E (1 + 2 ln V) of |dL/dH| p / T
        lnS = lse - z.double().amax(-1) / t
        extra = 2 * ref.E * (1 + lnS.abs() + (lnS - H).abs()) * b.double().abs() / t
        ref.close_grad(grad, want, size + (extra[:, None] * p) / (2 * ref.R), rel=2 * ref.R)


@pytest.mark.parametrize("T", [1e20, 1e28, 1e30, 1e33])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,V", LAUNCHES)
def test_masked_logits_at_the_highest_temperatures(torch, n, V, T, dtype):  # noqa: F811
    """Every logit left counts the same: H is the logarithm of their number, l its negative; a logit of -inf stays out."""
    dt = getattr(torch, dtype)
    z, tok, g = logits(torch, n, V, dt, V)
    z[:, 1::3] = float("-inf")
    tok = (tok // 3) * 3
    ctx = context(V, dt, T)
    T = float(torch.tensor(T, dtype=torch.float32))          # as the context holds it
    lp, ent, lo, only = out(torch, n, 4)
    ctx.token_logprob(z, tok, lp, ent, lo)
    ctx.token_logprob(z, tok, only)
    lnp, p, l, H, lse, on = ref.rows(z, tok, T)
    assert int((p[0] > 0).sum()) == V - (V + 1) // 3
    for got in (lp, only):
        ref.close_logp(got, l)
    ref.close_logp(lo, lse)
    ref.close_entropy(ent, H, lse)
    a, b = torch.randn(n, generator=g, device="cuda") * T, torch.randn(n, generator=g, device="cuda") * T
    grad = torch.full_like(z, 9.0)
    ctx.token_logprob_grad(z, tok, a, grad, grad_entropy=b)
    assert bool((grad[:, 1::3] == 0).all()) and ctx.status() == 0
    want, size = ref.gradient(lnp, p, H, tok, on, a.double(), b.double(), T)
    extra = 2 * ref.E * (1 + 2 * H.abs()) * b.double().abs() / T
    ref.close_grad(grad, want, size + (extra[:, None] * p) / ref.R)


@pytest.mark.parametrize("smoothing", [0.0, 0.1, 0.5])
@pytest.mark.parametrize("where", ["chosen", "rejected", "both"])
def test_preference_of_tokens_of_probability_zero(torch, where, smoothing):  # noqa: F811
    """A counted token whose logit is -inf: a sequence's log-prob of -inf, and the loss that the formula gives."""
    V, n = 50, 6
    z, tok, _ = logits(torch, n, V, torch.float32, 9)
    if where != "rejected":
        z[0, tok[0].long()] = float("-inf")                  # pair 0 (rows 0, 1 against 3, 4); pair 1 (row 2 against 5) is ordinary
    if where != "chosen":
        z[4, tok[4].long()] = float("-inf")
    start = torch.tensor([0, 2, 3, 5, 6], dtype=torch.int32, device="cuda")
    ctx = context(V, torch.float32)
    for refs in (None, torch.zeros(4, device="cuda")):
        so, po, total = out(torch, 4) + out(torch, 2) + out(torch, 1)
        scratch = torch.empty(16 * n, dtype=torch.uint8, device="cuda")
        grad = torch.full_like(z, 9.0)
        ctx.preference_loss(z, tok, start, po, so, scratch, ref_logp=refs, label_smoothing=smoothing, loss_out=total, grad_out=grad)
        assert ctx.status() == 0
        assert [float(v) == float("-inf") for v in so] == [where != "rejected", False, where != "chosen", False]
        u = {"chosen": -float("inf"), "rejected": float("inf"), "both": float("nan")}[where]
        # -(1 - s) ln sigma(u) - s ln sigma(-u), a factor of 0 making its term 0
        want = float("nan") if u != u else float("inf") if u < 0 or smoothing > 0 else 0.0
        assert str(float(po[0])) == str(want) and str(float(total)) == str(want if want != 0 else float(po[1]))
        assert 0.0 < float(po[1]) < 10.0
        # the slope is finite: beta (s - 1) at -inf, beta s at +inf
        if u == u:
            d = 0.1 * (smoothing - 1 if u < 0 else smoothing)
            assert float(grad[1, tok[1].long()]) == pytest.approx(d * (1 - float(torch.softmax(z[1], 0)[tok[1].long()])), rel=1e-4, abs=1e-9)
            assert bool(torch.isfinite(grad).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_temperatures_whose_reciprocal_32_bits_do_not_hold(torch, dtype):  # noqa: F811
    """1 / T beyond the range of 32 bits: refused, nothing is launched; the lowest temperature above is served."""
    import paper_2512_11280_b200 as adasd
    dt, V = getattr(torch, dtype), 1000
    z, tok, g = masked(torch, 5, V, dt, 1)
    z[:, 0] = 100.0
    tok[:3] = 0
    lp, ent, rl = out(torch, 5, 3)
    a = torch.full((5,), 0.1, device="cuda")
    grad = torch.full_like(z, 9.0)
    start = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    so, po, scratch = out(torch, 2)[0], out(torch, 1)[0], torch.empty(80, dtype=torch.uint8, device="cuda")
    ctx = context(V, dt, 4.2e-39)
    for call in (lambda: ctx.token_logprob(z, tok, lp), lambda: ctx.token_logprob_grad(z, tok, a, grad),
                 lambda: ctx.policy_loss(z, tok, a, rl, grad_out=grad), lambda: ctx.preference_loss(z, tok, start, po, so, scratch, grad_out=grad)):
        with pytest.raises(adasd.AdasdError) as e:
            call()
        assert e.value.code == adasd.ERR_SHAPE
    assert bool((lp == -7).all()) and bool((grad == 9).all()) and ctx.status() == 0
    ctx = context(V, dt, 4.3e-39)
    ctx.token_logprob(z, tok, lp, ent)
    assert bool((lp[:3] == 0).all()) and bool((ent == 0).all()) and bool((lp[3:] == float("-inf")).all())
    ctx.token_logprob_grad(z, tok, a, grad, grad_entropy=a)
    assert bool((grad[:3] == 0).all()) and bool(torch.isfinite(grad).all()) and ctx.status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [1, 7, 16])
def test_many_short_rows(torch, V, dtype):  # noqa: F811
    """Rows of a unit or two, 300000 of them: log-probs, gradients, a preference loss of two long pairs."""
    dt, n = getattr(torch, dtype), 300000
    z, tok, g = logits(torch, n, V, dt, V)
    tok[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
    ctx = context(V, dt)
    lnp, p, l, H, lse, on = ref.rows(z, tok)
    lp, ent = out(torch, n, 2)
    ctx.token_logprob(z, tok, lp, ent)
    ref.close_logp(lp, l)
    ref.close_entropy(ent, H, torch.where(on, lse - z.double().amax(-1), 0.0))
    a, b = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    want, size = ref.gradient(lnp, p, H, tok, on, a.double(), b.double(), 1.0)
    for off in (0, 1):                                       # the gradient where the logits lie relative to 16 bytes, and elsewhere
        buf = torch.full((n * V + 64,), 9.0, dtype=dt, device="cuda")
        grad = buf[off:off + n * V].view(n, V)
        ctx.token_logprob_grad(z, tok, a, grad, grad_entropy=b)
        ref.close_grad(grad, want, size)
        assert bool((buf[:off] == 9.0).all()) and bool((buf[off + n * V:] == 9.0).all())
    start = torch.tensor([0, n // 5, n // 2, n // 2, n], dtype=torch.int32, device="cuda")
    so, po, scratch = out(torch, 4)[0], out(torch, 2)[0], torch.empty(16 * n, dtype=torch.uint8, device="cuda")
    grad = torch.full_like(z, 9.0)
    ctx.preference_loss(z, tok, start, po, so, scratch, rule="hinge", beta=1e-7, average=True, grad_out=grad)
    counts = [max(1, int(on[start[s]:start[s + 1]].sum())) for s in range(4)]
    dl = torch.zeros(n, dtype=torch.float64, device="cuda")
    beta = float(torch.tensor(1e-7))
    for s in range(4):
        dl[start[s]:start[s + 1]] = (-beta if s < 2 else beta) / counts[s]
    want, size = ref.gradient(lnp, p, H, tok, on, torch.where(on, dl, 0.0), 0 * dl, 1.0)
    ref.close_grad(grad, want, size)
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,V", [(500, 5003), (60, 50257), (50, 131080)])
def test_a_slice_of_padded_logits_and_a_dense_gradient(torch, n, V, dtype):  # noqa: F811
    """logits[:, :V] of rows padded to a multiple of 64, the gradient [n, V]: they lie differently relative to 16 bytes."""
    dt = getattr(torch, dtype)
    pad = -(-(V + 1) // 64) * 64
    z, tok, g = logits(torch, n, pad, dt, V)
    z[:, V:] = float("nan")
    tok = tok % V
    tok[::5] = -1
    z = z[:, :V]
    ctx = context(V, dt, 0.8)
    t = float(torch.tensor(0.8, dtype=torch.float32))
    lnp, p, l, H, lse, on = ref.rows(z, tok, t)
    A, rl, grad = torch.randn(n, generator=g, device="cuda"), out(torch, n)[0], torch.full((n, V), 9.0, dtype=dt, device="cuda")
    for coef in (0.0, 0.3):
        ctx.policy_loss(z, tok, A, rl, entropy_coef=coef, grad_out=grad)
        want, size = ref.gradient(lnp, p, H, tok, on, torch.where(on, -A.double(), 0.0), torch.full_like(l, -coef), t)
        ref.close_grad(grad, want, size)
    start = torch.tensor([0, n // 2, n], dtype=torch.int32, device="cuda")
    so, po, scratch = out(torch, 2)[0], out(torch, 1)[0], torch.empty(16 * n, dtype=torch.uint8, device="cuda")
    ctx.preference_loss(z, tok, start, po, so, scratch, rule="hinge", beta=1e-4, grad_out=grad)
    beta = float(torch.tensor(1e-4))
    dl = torch.where(torch.arange(n, device="cuda") < n // 2, -beta, beta).double()
    want, size = ref.gradient(lnp, p, H, tok, on, torch.where(on, dl, 0.0), 0 * dl, t)
    ref.close_grad(grad, want, size)
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,V", [(100, 32000), (100, 151936), (60, 600000), (4, 600000)])
def test_accuracy_as_stated(torch, n, V, dtype):  # noqa: F811
    """ln S within (V / 256 + 128) 2^-24, p_v within that and (4 |ln p_v| + 8) 2^-24 of itself, on rows whose sums round the same way
    again and again: rising logits (every group of units has a new largest one), equal ones, one far above the others."""
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.linspace(-4, 4, V, device="cuda")[None].repeat(n, 1)
    z[1::3] = -3 * torch.rand(len(range(1, n, 3)), 1, generator=g, device="cuda")
    z[2::3] = -10.0
    z[:, 7] = 5.0
    z = (z + torch.rand(n, 1, generator=g, device="cuda")).to(dt)
    tok = torch.full((n,), V // 2, dtype=torch.int32, device="cuda")
    ctx = context(V, dt)
    lnp, p, l, H, lse, on = ref.rows(z, tok)
    S = (V / 256 + 128) * ref.U32
    lp, ent, lo = out(torch, n, 3)
    ctx.token_logprob(z, tok, lp, ent, lo)
    assert bool(((lp.double() - l).abs() <= S + ref.U32 * l.abs()).all())
    assert bool(((lo.double() - lse).abs() <= S + ref.U32 * lse.abs()).all())
    grad = torch.full_like(z, 9.0)
    ctx.token_logprob_grad(z, tok, -torch.ones(n, device="cuda"), grad)      # p_v, the token's own less 1
    got = grad.double()
    got[:, V // 2] = p[:, V // 2]
    tol = p * (S + (4 * lnp.abs() + 8) * ref.U32 + (2.7e-6 if dt is torch.bfloat16 else 0.0))
    tol = tol + torch.finfo(dt).eps / 2 * (p + tol)
    assert bool(((got - p).abs() <= tol).all()), float(((got - p).abs() / tol).max())
    assert ctx.status() == 0
