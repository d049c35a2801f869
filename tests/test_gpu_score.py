"""Log-probs of given tokens, policy and preference losses, and their gradients, against 64 bits."""
import math

import pytest

from tests import score_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return torch


_ctx = {}


def context(V, dtype, T=1.0):
    import torch
    import paper_2512_11280_b200 as adasd
    key = (V, dtype)
    if key not in _ctx:
        _ctx[key] = adasd.Context(1, V, 1, adasd.ADASD_BF16 if dtype is torch.bfloat16 else adasd.ADASD_FP32, list_capacity=1)
    _ctx[key].set_warpers(T)
    return _ctx[key]


def gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def strided(torch, values, offset=0, pad=0, fill=7.0):
    """The values as rows that start `offset` elements into an allocation, `pad` elements apart; the whole buffer too."""
    n, V = values.shape
    buf = torch.full((offset + n * (V + pad) + 64,), fill, dtype=values.dtype, device="cuda")
    view = buf[offset:offset + n * (V + pad)].view(n, V + pad)[:, :V]
    view.copy_(values)
    return view, buf


def logits(torch, n, V, dtype, seed, scale=3.0):
    g = gen(torch, seed)
    z = (torch.randn(n, V, generator=g, device="cuda") * scale).to(dtype)
    tok = torch.randint(0, V, (n,), generator=g, device="cuda").int()
    return z, tok, g


def out(torch, n, k=1, fill=-7.0):
    return [torch.full((n,), fill, device="cuda") for _ in range(k)]


# One unit, edges of units, of a CTA of 2 warps (256 units), of a thread's 4, 8, 16 units, of a cluster; rows longer than a cluster
# holds (fp32 131072, bf16 262144 logits)
SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (1, 1000), (6, 2047), (3, 2056), (2, 4099), (300, 8200), (1, 32000), (300, 32000),
         (310, 33003), (3, 50257), (2, 128256), (90, 128256), (2, 151936)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,V", SIZES + [(2, 131073), (2, 262145), (2, 300001)])
def test_logprob_entropy_and_gradient(torch, n, V, dtype):
    dt = getattr(torch, dtype)
    z, tok, g = logits(torch, n, V, dt, 7 * n + V)
    for T in (1.0, 0.7):
        ctx = context(V, dt, T)
        lnp, p, l, H, lse, on = ref.rows(z, tok, T)
        lp, ent, lo = out(torch, n, 3)
        ctx.token_logprob(z, tok, lp, ent, lo)
        lnS = lse - z.double().amax(-1) / T
        ref.close_logp(lp, l)
        ref.close_logp(lo, lse)
        ref.close_entropy(ent, H, lnS)
        only, = out(torch, n)
        ctx.token_logprob(z, tok, only)                      # without the entropy: another kernel
        ref.close_logp(only, l)
        a, b = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
        for dH in (None, b):
            grad = torch.full_like(z, 9.0)
            ctx.token_logprob_grad(z, tok, a, grad, grad_entropy=dH)
            want, size = ref.gradient(lnp, p, H, tok, on, a.double(), torch.zeros_like(l) if dH is None else b.double(), T)
            ref.close_grad(grad, want, size)
        assert ctx.status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [1, 7, 1001, 4096, 33000, 140001])
@pytest.mark.parametrize("where", [(0, 0, 8, 8), (1, 0, 1, 0), (3, 1, 3, 1), (1, 3, 2, 0), (0, 1, 5, 1), (8, 8, 3, 5)])
def test_any_alignment_and_stride_and_nothing_beside_the_rows(torch, V, dtype, where):
    """Offsets and gaps (elements) of the logits and of the gradient; what lies between and around the rows stays."""
    dt = getattr(torch, dtype)
    n = 5
    values, tok, g = logits(torch, n, V, dt, V)
    tok[1] = -1                                              # a row left out among them
    z, zbuf = strided(torch, values, where[0], where[1], fill=float("nan"))
    grad, gbuf = strided(torch, torch.zeros_like(values), where[2], where[3])
    before = zbuf.clone()
    ctx = context(V, dt)
    lnp, p, l, H, lse, on = ref.rows(values, tok)
    lp, ent = out(torch, n, 2)
    ctx.token_logprob(z, tok, lp, ent)
    ref.close_logp(lp, l)
    ref.close_entropy(ent, H, torch.where(on, lse - values.double().amax(-1), 0.0))
    a, b = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    ctx.token_logprob_grad(z, tok, a, grad, grad_entropy=b)
    want, size = ref.gradient(lnp, p, H, tok, on, a.double(), b.double(), 1.0)
    ref.close_grad(grad, want, size)
    inside = torch.zeros_like(gbuf, dtype=torch.bool)
    inside[where[2]:where[2] + n * (V + where[3])].view(n, V + where[3])[:, :V] = True
    assert bool((gbuf[~inside] == 7.0).all())
    assert torch.equal(before.nan_to_num(3.0), zbuf.nan_to_num(3.0))
    # a preference loss writes its gradient by another kernel
    start = torch.tensor([0, 3, n], dtype=torch.int32, device="cuda")
    gbuf.fill_(7.0)
    preference(torch, ctx, z, values, tok, start, grad, "sigmoid")
    assert bool((gbuf[~inside] == 7.0).all())
    # in place: the logits become the gradient
    z.copy_(values)
    ctx.token_logprob_grad(z, tok, a, z, grad_entropy=b)
    ref.close_grad(z, want, size)
    assert ctx.status() == 0


def policy(torch, ctx, z, values, tok, g, T=1.0, old=True, kl=0.1, ent=0.05, weight=True, grad=None, scale=0.5, forward_only=False):
    n = z.shape[0]
    lnp, p, l, H, lse, on = ref.rows(values, tok, T)
    rnd = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    A, d, r = rnd(), 0.3 * rnd().double(), 0.4 * rnd()
    for edge in (0.8, 1.3):                                  # (on the very edge of the clip range either branch may hold)
        d = torch.where((torch.exp(-d) - edge).abs() < 1e-3, d + 0.01, d)
    A[0] = 0.0
    o = (l + d).float() if old else None
    rf = (l + r).float() if kl else None
    w = torch.rand(n, generator=g, device="cuda") if weight else None
    if w is not None:
        w[-1] = 0.0 if n > 1 else 1.0
    loss, k3, dl, dH, size, dsize, on = ref.policy(l, H, on, A, o, rf, w, 0.2, 0.3, kl, ent, scale)
    row_loss, total, lp, eo, ko = out(torch, n) + out(torch, 1) + out(torch, n, 3)
    grad = None if forward_only else torch.full_like(z, 9.0) if grad is None else grad
    ctx.policy_loss(z, tok, A, row_loss, old_logp=o, ref_logp=rf, weight=w, clip_low=0.2, clip_high=0.3, kl_coef=kl, entropy_coef=ent,
                    scale=scale, loss_out=total, logp_out=lp, entropy_out=eo if ent else None, kl_out=ko if kl else None, grad_out=grad)
    tol = 4 * ref.E * size + ref.U32 * loss.abs()
    assert bool(((row_loss.double() - loss).abs() <= tol).all()), float(((row_loss.double() - loss).abs() / tol).max())
    assert abs(float(total) - float(loss.sum())) <= float(tol.sum() + ref.U32 * loss.sum().abs()) + 1e-30
    ref.close_logp(lp, torch.where(on, l, 0.0))
    if kl:
        assert bool(((ko.double() - k3).abs() <= 4 * ref.E * (torch.exp(r.double()) + 1) + ref.U32 * k3).all())
    if not forward_only:
        want, gsize = ref.gradient(lnp, p, H, tok, on, dl, dH, T)
        _, gsize = ref.gradient(lnp, p, H, tok, on, dsize, dH, T)
        ref.close_grad(grad, want, gsize)
    return row_loss, grad


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,V", SIZES)
def test_policy_loss(torch, n, V, dtype):
    dt = getattr(torch, dtype)
    z, tok, g = logits(torch, n, V, dt, 5 * n + V)
    tok[n // 2] = V if n > 2 else tok[n // 2]                # left out
    ctx = context(V, dt, 1.0)
    policy(torch, ctx, z, z, tok, g)
    policy(torch, ctx, z, z, tok, g, old=False, kl=0.0, ent=0.0, weight=False)
    policy(torch, ctx, z, z, tok, g, forward_only=True)
    context(V, dt, 1.4)
    policy(torch, ctx, z, z, tok, g, T=1.4, ent=0.0)
    assert ctx.status() == 0


def preference(torch, ctx, z, values, tok, start, grad, rule, T=1.0, refs=True, pw=None, average=False, margin=0.25, beta=0.3, seed=3):
    n, P = z.shape[0], (start.numel() - 1) // 2
    g = gen(torch, seed)
    lnp, p, l, H, lse, on = ref.rows(values, tok, T)
    st = [min(max(v, 0), n) for v in start.tolist()]
    seq, *_ = ref.preference(l, on, st, None, pw, rule, beta, margin, 0.0, average, 1.0)
    r = (seq + 2 * torch.randn(2 * P, generator=g, device="cuda").double()).float() if refs else None
    smooth = 0.1 if rule == "sigmoid" else 0.0
    seq, loss, dl, dD = ref.preference(l, on, st, r, pw, rule, beta, margin, smooth, average, 0.5)
    so, po, total = out(torch, 2 * P) + out(torch, P) + out(torch, 1)
    scratch = torch.full((16 * n + 64,), 255, dtype=torch.uint8, device="cuda")
    ctx.preference_loss(z, tok, start, po, so, scratch, ref_logp=r, pair_weight=pw, rule=rule, beta=beta, margin=margin,
                        label_smoothing=smooth, average=average, scale=0.5, loss_out=total, grad_out=grad)
    # a sequence's sum is its rows' E and the rounding of z_x - m off; the loss's slope carries that over
    rows = max([1] + [st[s + 1] - st[s] for s in range(2 * P)])
    per = (ref.E + 2 * ref.U32 * float(l.abs().max() + lse.abs().max())) * (1 if average else rows)
    assert bool(((so.double() - seq).abs() <= per + ref.U32 * seq.abs()).all())
    curve = 2 * per * (dD.abs() + 2 * per + beta * beta)
    assert bool(((po.double() - loss).abs() <= curve + 2 * ref.U32 * loss.abs()).all()), (po, loss)
    assert abs(float(total) - float(loss.sum())) <= float((curve + 2 * ref.U32 * loss.abs()).sum()) + 1e-30
    if grad is not None:
        inside = torch.zeros(n, dtype=torch.bool, device="cuda")
        inside[st[0]:max(st)] = True
        want, size = ref.gradient(lnp, p, H, tok, on, dl, torch.zeros_like(l), T)
        slope = 2 * per * (2.0 if rule == "squared" else beta * beta)       # of dL/dl
        if rule == "hinge":
            slope = 0.0
        ref.close_grad(grad[inside], want[inside], size[inside] + (slope / ref.R) * (size[inside] > 0))
    return so, po


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rule", ["sigmoid", "squared", "hinge"])
@pytest.mark.parametrize("V", [1, 9, 2047, 8200, 50257, 151936])
def test_preference_loss(torch, V, rule, dtype):
    dt = getattr(torch, dtype)
    n = 23
    z, tok, g = logits(torch, n, V, dt, V)
    tok[[2, 9, 10, 22]] = torch.tensor([-1, -100, V, -1], dtype=torch.int32, device="cuda")
    ctx = context(V, dt)
    # three pairs: a sequence of one row, one of none, one with no row that counts (9, 10); rows ahead and behind stay
    start = torch.tensor([1, 4, 5, 9, 9, 11, 21], dtype=torch.int32, device="cuda")
    grad = torch.full_like(z, 9.0)
    preference(torch, ctx, z, z, tok, start, grad, rule)
    assert bool((grad[:1] == 9.0).all()) and bool((grad[21:] == 9.0).all())
    preference(torch, ctx, z, z, tok, start, grad, rule, average=True, refs=False)
    pw = torch.tensor([0.5, 0.0, 2.0], device="cuda")
    preference(torch, ctx, z, z, tok, start, grad, rule, pw=pw)
    assert bool((grad[4] == 0).all())                        # pair 1 has weight 0: its chosen sequence is row 4
    preference(torch, ctx, z, z, tok, start, None, rule)
    context(V, dt, 0.6)
    preference(torch, ctx, z, z, tok, start, grad, rule, T=0.6)
    assert ctx.status() == 0


@pytest.mark.parametrize("average", [False, True])
def test_preference_of_long_sequences(torch, average):
    """More rows than a CTA's threads, a sequence in 64-bit sums."""
    n, V = 1500, 1000
    z, tok, g = logits(torch, n, V, torch.bfloat16, 1)
    start = torch.tensor([0, 700, 1500], dtype=torch.int32, device="cuda")
    preference(torch, context(V, torch.bfloat16), z, z, tok, start, torch.empty_like(z), "squared", average=average, beta=0.05)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [40, 5000, 140000, 270000])
def test_masked_logits_and_extreme_rows(torch, V, dtype):
    dt = getattr(torch, dtype)
    low = torch.finfo(dt).min
    z, tok, g = logits(torch, 9, V, dt, V)
    half = V // 2
    z[0, half:] = float("-inf")                              # half of the vocabulary masked, by -inf and by the lowest value
    z[1, :half] = low
    z[2, 1:] = float("-inf")                                 # one token left: l = 0, H = 0
    z[3] += 5000.0                                           # a large offset
    z[4] = 0.0                                               # flat
    z[5] = -1e30 if dt is torch.float32 else low             # (rows 5 to 8: no finite logit to speak of, NaN, +inf, all -inf)
    z[6, V - 1] = float("nan")
    z[7, half] = float("inf")
    z[8] = float("-inf")
    tok[0], tok[1], tok[2] = 3, V - 1, 0
    ctx = context(V, dt)
    ok = slice(0, 5)
    lnp, p, l, H, lse, on = ref.rows(z, tok)
    lp, ent, lo = out(torch, 9, 3)
    ctx.token_logprob(z, tok, lp, ent, lo)
    assert ctx.status() == 4                                 # ADASD_STATUS_NAN
    # (logits near 5000 in bf16 or fp32 are exact: so is their difference to the largest)
    ref.close_logp(lp[ok], l[ok])
    ref.close_logp(lo[ok], lse[ok])
    ref.close_entropy(ent[ok], H[ok], (lse - z.double().amax(-1))[ok])
    assert float(lp[2]) == 0.0 and float(ent[2]) == 0.0
    for t in (lp, ent, lo):
        assert bool(t[5:].isnan().all()), t
    a, b = torch.randn(9, generator=g, device="cuda"), torch.randn(9, generator=g, device="cuda")
    for dH in (None, b):
        grad = torch.zeros_like(z)
        ctx.token_logprob_grad(z, tok, a, grad, grad_entropy=dH)
        assert ctx.status() == 4
        want, size = ref.gradient(lnp[ok], p[ok], H[ok], tok[ok], on[ok], a[ok].double(), (0 * b if dH is None else b)[ok].double(), 1.0)
        ref.close_grad(grad[ok], want, size)
        assert bool(grad[5:].isnan().all())
        assert bool((grad[0, half:] == 0).all()) and bool((grad[1, :half] == 0).all())
    # unusable rows that are left out, by token or by weight, are not read
    skip = tok.clone()
    skip[5:7] = -1
    w = torch.ones(9, device="cuda")
    w[7:] = 0
    rl, total, grad = out(torch, 9)[0], out(torch, 1)[0], torch.full_like(z, 9.0)
    ctx.policy_loss(z, skip, a, rl, weight=w, loss_out=total, grad_out=grad, entropy_coef=0.1)
    assert ctx.status() == 0 and bool(torch.isfinite(total).all()) and bool((grad[5:] == 0).all()) and bool((rl[5:] == 0).all())
    ctx.policy_loss(z, tok, a, rl, loss_out=total, grad_out=grad)
    assert ctx.status() == 4 and bool(total.isnan()) and bool(rl[5:].isnan().all()) and bool(grad[5:].isnan().all())
    assert not bool(rl[:5].isnan().any()) and not bool(grad[:5].isnan().any())
    # a pair with such rows is NaN, a pair of weight 0 with them is nothing
    start = torch.tensor([0, 2, 3, 5, 9], dtype=torch.int32, device="cuda")      # pairs (0-1, 3-4) and (2, 5-8)
    scratch = torch.empty(16 * 9, dtype=torch.uint8, device="cuda")
    so, po = out(torch, 4)[0], out(torch, 2)[0]
    ctx.preference_loss(z, tok, start, po, so, scratch, loss_out=total, grad_out=grad)
    assert ctx.status() == 4 and bool(po[1].isnan()) and bool(total.isnan()) and bool(torch.isfinite(po[0]))
    assert bool(grad[2].isnan().all()) and bool(grad[5:].isnan().all()) and not bool(grad[[0, 1, 3, 4]].isnan().any())
    pw = torch.tensor([1.0, 0.0], device="cuda")
    ctx.preference_loss(z, tok, start, po, so, scratch, pair_weight=pw, loss_out=total, grad_out=grad)
    assert ctx.status() == 4 and bool(torch.isfinite(total)) and float(po[1]) == 0.0
    assert bool((grad[2] == 0).all()) and bool((grad[5:] == 0).all())


def test_token_of_probability_zero(torch):
    """A token whose own logit is -inf: l = -inf, the ratio 0, the KL estimate infinite; the gradient of the ratio is 0."""
    V = 100
    z, tok, g = logits(torch, 3, V, torch.float32, 2)
    z[torch.arange(3), tok.long()] = float("-inf")
    ctx = context(V, torch.float32)
    lp, = out(torch, 3)
    ctx.token_logprob(z, tok, lp)
    assert bool((lp == float("-inf")).all()) and ctx.status() == 0
    A, old = torch.tensor([1.0, -2.0, 0.0], device="cuda"), torch.full((3,), -1.0, device="cuda")
    rl, kl, grad = out(torch, 3)[0], out(torch, 3)[0], torch.full_like(z, 9.0)
    ctx.policy_loss(z, tok, A, rl, old_logp=old, ref_logp=old, kl_out=kl, grad_out=grad)
    assert rl.tolist() == [0.0, pytest.approx(1.6), 0.0] and bool((grad == 0).all()) and bool((kl == math.inf).all())


def test_ratios_that_overflow(torch):
    V = 64
    z, tok, g = logits(torch, 3, V, torch.float32, 4)
    ctx = context(V, torch.float32)
    old = torch.full((3,), -1e5, device="cuda")
    A = torch.tensor([1.0, 0.0, -1.0], device="cuda")
    rl, grad = out(torch, 3)[0], torch.full_like(z, 9.0)
    ctx.policy_loss(z, tok, A, rl, old_logp=old, clip_high=0.28, grad_out=grad)
    assert float(rl[0]) == pytest.approx(-1.28) and float(rl[1]) == 0.0 and float(rl[2]) == math.inf
    assert bool((grad[:2] == 0).all())


@pytest.mark.parametrize("n,V,dtype", [(4, 1000, "float32"), (2, 50257, "float32"), (2, 140001, "float32")])
def test_gradients_against_differences(torch, n, V, dtype):
    """Along random directions: (L(z + h d) - L(z - h d)) / 2h, L as the device reports it."""
    dt = getattr(torch, dtype)
    z, tok, g = logits(torch, n, V, dt, 11)
    ctx = context(V, dt, 0.9)
    lp, = out(torch, n)
    ctx.token_logprob(z, tok, lp)
    rnd = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    A, old, rf = rnd(), lp + 0.05, lp + 0.3 * rnd()
    start = torch.tensor([0, n // 2, n], dtype=torch.int32, device="cuda")
    scratch = torch.empty(16 * n, dtype=torch.uint8, device="cuda")

    def pol(y, grad=None):
        rl, = out(torch, n)
        ctx.policy_loss(y, tok, A, rl, old_logp=old, ref_logp=rf, kl_coef=0.3, entropy_coef=0.2, grad_out=grad)
        return rl.double().sum()

    def pre(y, grad=None):
        so, po = out(torch, 2)[0], out(torch, 1)[0]
        ctx.preference_loss(y, tok, start, po, so, scratch, beta=0.2, grad_out=grad)
        return po.double().sum()
    for loss in (pol, pre):
        grad = torch.empty_like(z)
        loss(z, grad)
        for k in range(3):
            d = torch.randn(z.shape, generator=g, device="cuda")
            d[torch.arange(n), tok.long()] += 3.0
            h = 2.0 ** -6
            num = (loss(z + h * d) - loss(z - h * d)) / (2 * h)
            an = (grad.double() * d.double()).sum()
            # values of size up to 10 n rounded at 2^-24 over 2 h; the third derivative times h^2 / 6
            assert abs(float(num - an)) <= 10 * n * 2.0 ** -24 / h + 30 * h * h * n, (float(num), float(an))


def test_they_run_together(torch):
    """Score with a reference and a behaviour model, train by each loss: the losses' log-probs are those of the scoring call, their
    gradients those of its backward pass."""
    n, V = 40, 5003
    dt = torch.bfloat16
    z, tok, g = logits(torch, n, V, dt, 21)
    z_ref, z_old = ((z.float() + 0.2 * torch.randn(z.shape, generator=g, device="cuda")).to(dt) for _ in range(2))
    tok[5] = -100
    ctx = context(V, dt, 0.8)
    lp, lr, lo, lp2, kl, rl = out(torch, n, 6)
    for y, o in ((z, lp), (z_ref, lr), (z_old, lo)):
        ctx.token_logprob(y, tok, o)
    A = torch.randn(n, generator=g, device="cuda")
    grad, again = torch.empty_like(z), torch.empty_like(z)
    ctx.policy_loss(z, tok, A, rl, old_logp=lo, ref_logp=lr, kl_coef=0.2, logp_out=lp2, kl_out=kl, grad_out=grad)
    # (either call is its tolerance off the truth at the most; they may sum in different orders)
    assert bool(((lp.double() - lp2.double()).abs() <= 2 * (ref.E + ref.U32 * lp.double().abs())).all())
    l = lp.double().requires_grad_(True)
    ratio, r = torch.exp(l - lo.double()), lr.double() - l
    loss = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A) + 0.2 * (torch.exp(r) - r - 1)
    dl, = torch.autograd.grad(loss[tok >= 0].sum(), l)
    ctx.token_logprob_grad(z, tok, dl.float(), again)
    d = (grad.float() - again.float()).abs()
    assert float((d / (again.float().abs() + 1e-6)).max()) <= 2.0 ** -7      # a step of bf16: the coefficient rounded once more
    start = torch.tensor([0, 7, 20, 33, 40], dtype=torch.int32, device="cuda")
    so, sr, po = out(torch, 4) + out(torch, 4) + out(torch, 2)
    scratch = torch.empty(16 * n, dtype=torch.uint8, device="cuda")
    ctx.preference_loss(z_ref, tok, start, po, sr, scratch)
    ctx.preference_loss(z, tok, start, po, so, scratch, ref_logp=sr, grad_out=grad)
    for s in range(4):
        assert abs(float(so[s]) - float(lp[start[s]:start[s + 1]].double().sum())) <= 1e-4
    assert ctx.status() == 0


def test_same_bits_every_time_on_streams_and_in_graphs(torch):
    n, V = 64, 33003
    z, tok, g = logits(torch, n, V, torch.bfloat16, 31)
    ctx = context(V, torch.bfloat16)
    A = torch.randn(n, generator=g, device="cuda")
    start = torch.tensor([0, 20, 64], dtype=torch.int32, device="cuda")

    class Call:
        def __init__(self, y):
            self.y = y
            self.rl, self.t1, self.so, self.po, self.t2 = (out(torch, k)[0] for k in (n, 1, 2, 1, 1))
            self.g1, self.g2 = torch.zeros_like(y), torch.zeros_like(y)
            self.scratch = torch.empty(16 * n, dtype=torch.uint8, device="cuda")

        def run(self):
            ctx.policy_loss(self.y, tok, A, self.rl, entropy_coef=0.1, loss_out=self.t1, grad_out=self.g1)
            ctx.preference_loss(self.y, tok, start, self.po, self.so, self.scratch, loss_out=self.t2, grad_out=self.g2)

        def same(self, o):
            return all(torch.equal(getattr(self, k), getattr(o, k)) for k in ("rl", "t1", "so", "po", "t2", "g1", "g2"))

    y2 = (z.float() * 0.5).to(z.dtype)
    want, want2 = Call(z), Call(y2)
    want.run(), want2.run()
    torch.cuda.synchronize()
    # two streams at once, one context
    a, b, s1, s2 = Call(z), Call(y2), torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s1):
            a.run()
        with torch.cuda.stream(s2):
            b.run()
    torch.cuda.synchronize()
    assert a.same(want) and b.same(want2)
    # a captured graph, its inputs changed between replays
    c = Call(z.clone())
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.run()
        for y, w in ((y2, want2), (z, want)):
            c.y.copy_(y)
            graph.replay()
            s.synchronize()
            assert c.same(w)
    assert ctx.status() == 0


@pytest.mark.parametrize("n,V", [(5, 999), (400, 45003), (400, 9001), (400, 70000)])
def test_first_call_inside_a_capture(torch, n, V):
    """Nothing has to be called before a capture: what a launch looks up for itself the first time is allowed there."""
    z, tok, g = logits(torch, n, V, torch.bfloat16, 51)
    ctx = context(V, torch.bfloat16)
    A = torch.randn(n, generator=g, device="cuda")
    rl, lp = out(torch, n, 2)
    grad = torch.empty_like(z)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.token_logprob(z, tok, lp)
        ctx.policy_loss(z, tok, A, rl, grad_out=grad)
    graph.replay()
    torch.cuda.synchronize()
    lnp, p, l, H, lse, on = ref.rows(z, tok)
    ref.close_logp(lp, l)
    want, size = ref.gradient(lnp, p, H, tok, on, -A.double(), torch.zeros_like(l), 1.0)
    ref.close_grad(grad, want, size)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [9, 4100, 9001, 33003, 50264])
def test_many_rows_many_left_out(torch, V, dtype):
    """Most rows left out, runs of them longer than what is looked at at once, the last ones too; nothing of them is read."""
    dt = getattr(torch, dtype)
    n = 3000 if V < 10000 else 1000
    z, tok, g = logits(torch, n, V, dt, V)
    keep = torch.rand(n, generator=g, device="cuda") < 0.2
    keep[200:260] = False
    keep[-3:] = False
    z[~keep] = float("nan")
    tok = torch.where(keep, tok, -100)
    ctx = context(V, dt)
    clean = torch.where(keep[:, None], z, torch.zeros_like(z))
    lnp, p, l, H, lse, on = ref.rows(clean, tok)
    lp, ent, rl = out(torch, n, 3)
    ctx.token_logprob(z, tok, lp, ent)
    ref.close_logp(lp, l)
    assert bool((ent[~keep] == 0).all())
    A = torch.randn(n, generator=g, device="cuda")
    for coef in (0.0, 0.3):
        grad = torch.full_like(z, 9.0)
        ctx.policy_loss(z, tok, A, rl, entropy_coef=coef, grad_out=grad)
        want, size = ref.gradient(lnp, p, H, tok, on, -A.double(), torch.full_like(l, -coef), 1.0)
        ref.close_grad(grad, want, size)
        assert bool((grad[~keep] == 0).all()) and bool((rl[~keep] == 0).all())
        ctx.policy_loss(z.clone(), torch.full_like(tok, -1), A, rl, entropy_coef=coef, grad_out=grad)       # nothing to do at all
        assert bool((grad == 0).all()) and bool((rl == 0).all())
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n,V", [(700, 900), (400, 8200), (400, 9001), (400, 20000), (300, 70001)])
def test_unusable_rows_among_many_and_gradients_in_place(torch, n, V, dtype):
    """NaN, +inf and rows without a finite logit spoil their own outputs alone; the logits may become the gradient."""
    dt = getattr(torch, dtype)
    z, tok, g = logits(torch, n, V, dt, n + V)
    bad = torch.randperm(n, generator=g, device="cuda")[:12]
    z[bad[:4], V // 3] = float("nan")
    z[bad[4:8], V - 1] = float("inf")
    z[bad[8:10]] = float("-inf")
    z[bad[10:]] = torch.finfo(dt).min
    fine = torch.ones(n, dtype=torch.bool, device="cuda")
    fine[bad] = False
    ctx = context(V, dt)
    lnp, p, l, H, lse, on = ref.rows(z[fine], tok[fine])
    lp, ent, rl = out(torch, n, 3)
    ctx.token_logprob(z, tok, lp, ent)
    assert ctx.status() == 4                                 # ADASD_STATUS_NAN
    ref.close_logp(lp[fine], l)
    assert bool(lp[~fine].isnan().all()) and bool(ent[~fine].isnan().all())
    A = torch.randn(n, generator=g, device="cuda")
    for coef in (0.0, 0.3):
        grad, here = torch.full_like(z, 9.0), z.clone()
        ctx.policy_loss(z, tok, A, rl, entropy_coef=coef, grad_out=grad)
        assert ctx.status() == 4
        want, size = ref.gradient(lnp, p, H, tok[fine], on, -A[fine].double(), torch.full_like(l, -coef), 1.0)
        ref.close_grad(grad[fine], want, size)
        assert bool(grad[~fine].isnan().all()) and bool(rl[~fine].isnan().all()) and not bool(rl[fine].isnan().any())
        ctx.policy_loss(here, tok, A, rl, entropy_coef=coef, grad_out=here)
        assert torch.equal(here.nan_to_num(5.0), grad.nan_to_num(5.0)) and ctx.status() == 4
    clean = z[fine]
    m = clean.shape[0]
    start = torch.tensor([0, m // 3, m], dtype=torch.int32, device="cuda")
    grad, here, scratch = torch.full_like(clean, 9.0), clean.clone(), torch.empty(16 * m, dtype=torch.uint8, device="cuda")
    so, po = out(torch, 2)[0], out(torch, 1)[0]
    ctx.preference_loss(clean, tok[fine], start, po, so, scratch, beta=1e-3, grad_out=grad)
    ctx.preference_loss(here, tok[fine], start, po, so, scratch, beta=1e-3, grad_out=here)
    assert torch.equal(here, grad) and ctx.status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T", [1e-3, 1e-7, 1e-9, 1e4])
@pytest.mark.parametrize("n,V", [(3, 5000), (400, 9001), (400, 20000)])
def test_temperatures_at_the_ends(torch, n, V, T, dtype):
    """Exponents (z - m) / T far beyond what 2^t resolves, and next to nothing; logits around 2000 and masks beside them."""
    dt = getattr(torch, dtype)
    z, tok, g = logits(torch, n, V, dt, V)
    z[: n // 2] += 2000.0
    z[:, 1::3] = float("-inf")
    z[:, 2::7] = -1e30
    tok = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, z.argmax(-1).int(), (tok // 21) * 21)     # (21 k: a logit)
    ctx = context(V, dt, T)
    T = float(torch.tensor(T, dtype=torch.float32))          # as the context holds it
    lnp, p, l, H, lse, on = ref.rows(z, tok, T)
    lp, = out(torch, n)
    ctx.token_logprob(z, tok, lp)
    # log2 e / T is held in 32 bits: exponents of size 1 and below, which alone count in S, are off by 2^-24 of it
    assert bool(((lp.double() - l).abs() <= ref.E + 4 * ref.U32 * l.abs()).all())
    a = torch.randn(n, generator=g, device="cuda")
    grad = torch.empty_like(z)
    ctx.token_logprob_grad(z, tok, a, grad)
    want, size = ref.gradient(lnp, p, H, tok, on, a.double(), torch.zeros_like(l), T)
    ref.close_grad(grad, want, size, rel=2 * ref.R)
    assert bool((grad[:, 1::3][z[:, 1::3] == float("-inf")] == 0).all()) and bool((grad[z <= -1e30] == 0).all())
    assert ctx.status() == 0


def test_offsets_beyond_32_bits(torch):
    """Rows far enough apart that offsets in elements and bytes pass 2^31 and 2^32."""
    V, n, stride = 1000, 3, (1 << 31) + 8
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 18 GB")
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((n, V), (stride, 1))
    gbuf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    grad = gbuf.as_strided((n, V), (stride, 1))
    values, tok, g = logits(torch, n, V, torch.bfloat16, 41)
    z.copy_(values)
    ctx = context(V, torch.bfloat16)
    policy(torch, ctx, z, values, tok, g, grad=grad)
    start = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
    preference(torch, ctx, z, values, tok, start, grad, "sigmoid")


def test_no_rows_no_pairs(torch):
    ctx = context(50, torch.float32)
    e = torch.empty(0, device="cuda")
    z, tok = torch.empty(0, 50, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    total = torch.full((1,), 5.0, device="cuda")
    ctx.token_logprob(z, tok, e)
    ctx.token_logprob_grad(z, tok, e, z)
    ctx.policy_loss(z, tok, e, e, loss_out=total, grad_out=z)
    assert float(total) == 0.0
    total.fill_(5.0)
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.preference_loss(z, tok, one, e, e, torch.empty(0, dtype=torch.uint8, device="cuda"), loss_out=total, grad_out=z)
    assert float(total) == 0.0
    # rows, but sequences of none
    z, tok, _ = logits(torch, 4, 50, torch.float32, 1)
    grad = torch.full_like(z, 9.0)
    so, po = out(torch, 2)[0], out(torch, 1)[0]
    ctx.preference_loss(z, tok, torch.zeros(3, dtype=torch.int32, device="cuda"), po, so, torch.empty(64, dtype=torch.uint8, device="cuda"),
                        loss_out=total, grad_out=grad)
    assert so.tolist() == [0.0, 0.0] and float(total) == pytest.approx(math.log(2)) and bool((grad == 9.0).all())


def test_refusals(torch):
    import paper_2512_11280_b200 as adasd
    V, n = 100, 4
    z, tok, _ = logits(torch, n, V, torch.bfloat16, 1)
    ctx = context(V, torch.bfloat16)
    f = lambda k=n: torch.zeros(k, device="cuda")  # noqa: E731
    scratch = torch.empty(16 * n, dtype=torch.uint8, device="cuda")
    start = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    grad = torch.zeros_like(z)

    def code(call):
        with pytest.raises(adasd.AdasdError) as e:
            call()
        return e.value.code

    lp = lambda **k: ctx.token_logprob(**{**dict(logits=z, tokens=tok, logp_out=f()), **k})  # noqa: E731
    pol = lambda **k: ctx.policy_loss(**{**dict(logits=z, tokens=tok, advantage=f(), row_loss_out=f()), **k})  # noqa: E731
    pre = lambda **k: ctx.preference_loss(**{**dict(logits=z, tokens=tok, seq_start=start, pair_loss_out=f(1), seq_logp_out=f(2),  # noqa: E731
                                                    scratch=scratch), **k})
    assert code(lambda: lp(tokens=tok.long())) == adasd.ERR_DTYPE
    assert code(lambda: lp(tokens=tok[:3])) == adasd.ERR_SHAPE
    assert code(lambda: lp(tokens=tok.cpu())) == adasd.ERR_DEVICE
    assert code(lambda: lp(logits=z.float())) == adasd.ERR_DTYPE
    assert code(lambda: lp(logits=z[:, :99])) == adasd.ERR_SHAPE
    assert code(lambda: lp(logits=z[0])) == adasd.ERR_SHAPE
    assert code(lambda: lp(logits=z.t().contiguous().t())) == adasd.ERR_SHAPE
    assert code(lambda: lp(logits=z[:1].expand(n, V))) == adasd.ERR_SHAPE
    assert code(lambda: lp(logp_out=f()[::2])) == adasd.ERR_SHAPE
    assert code(lambda: ctx.token_logprob_grad(z, tok, f(), grad[1:])) == adasd.ERR_SHAPE
    big = torch.zeros((n + 1) * V, dtype=z.dtype, device="cuda")
    assert code(lambda: ctx.token_logprob_grad(big[:n * V].view(n, V), tok, f(), big[1:n * V + 1].view(n, V))) == adasd.ERR_SHAPE
    assert code(lambda: pol(kl_coef=0.1)) == adasd.ERR_NULL
    assert code(lambda: pol(kl_out=f())) == adasd.ERR_NULL
    for k, bad in (("clip_low", (-0.1, 1.5, math.nan)), ("clip_high", (-0.1, math.inf, math.nan)), ("kl_coef", (-1.0, math.nan, math.inf)),
                   ("entropy_coef", (math.nan, math.inf)), ("scale", (math.nan, math.inf))):
        for v in bad:
            assert code(lambda: pol(**{k: v})) == adasd.ERR_SHAPE, (k, v)
    assert code(lambda: pre(rule="other")) == adasd.ERR_DTYPE
    assert code(lambda: pre(scratch=scratch[:-1])) == adasd.ERR_SHAPE
    assert code(lambda: pre(seq_start=start[:2])) == adasd.ERR_SHAPE
    assert code(lambda: pre(seq_logp_out=f(1))) == adasd.ERR_SHAPE
    for k, bad in (("beta", (0.0, -1.0, math.nan, math.inf)), ("margin", (math.nan,)), ("label_smoothing", (-0.1, 0.6, math.nan)),
                   ("scale", (math.inf,))):
        for v in bad:
            assert code(lambda: pre(**{k: v})) == adasd.ERR_SHAPE, (k, v)
    assert code(lambda: pre(rule="hinge", label_smoothing=0.1)) == adasd.ERR_SHAPE
    more = torch.empty(16 * n + 16, dtype=torch.uint8, device="cuda")
    assert code(lambda: pre(scratch=more[8:8 + 16 * n])) == adasd.ERR_ALIGN
    ctx.set_warpers(1.0, 5, 1.0)
    for call in (lp, pol, pre, lambda: ctx.token_logprob_grad(z, tok, f(), grad)):
        assert code(call) == adasd.ERR_DTYPE
    ctx.set_warpers(1.0, 0, 0.9)
    assert code(lp) == adasd.ERR_DTYPE
    ctx.set_warpers()
    s = torch.cuda.current_stream().cuda_stream
    assert adasd.adasd_token_logprob(ctx.handle, z.data_ptr(), V - 1, tok.data_ptr(), n, f().data_ptr(), None, None, s) == adasd.ERR_SHAPE
    assert adasd.adasd_token_logprob(ctx.handle, z.data_ptr(), V, tok.data_ptr(), -1, f().data_ptr(), None, None, s) == adasd.ERR_SHAPE
    assert adasd.adasd_token_logprob(ctx.handle, z.data_ptr() + 1, V, tok.data_ptr(), n, f().data_ptr(), None, None, s) == adasd.ERR_ALIGN
    assert adasd.adasd_token_logprob(ctx.handle, z.data_ptr(), V, tok.data_ptr() + 2, n, f().data_ptr(), None, None, s) == adasd.ERR_ALIGN
    torch.cuda.synchronize()
    assert ctx.status() == 0
