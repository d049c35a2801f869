"""Head calls at the edges of what the header allows."""
import pytest

from tests.head_reference import Head
from tests.test_gpu_head import context, inputs, out, scratch_for

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return torch


# ---- scratch ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("V,D", [(1, 8), (161, 64), (32000, 512), (32000, 2048), (128256, 2048), (50257, 1000), (300000, 136)])
def test_scratch_never_falls_with_rows(torch, V, D):
    ctx = context(V)
    last = [0, 0]
    for n in [*range(0, 700), *range(700, 9000, 31), *range(9000, 200000, 4801)]:
        now = [ctx.head_scratch(n, D, grad) for grad in (False, True)]
        assert now[0] >= last[0] and now[1] >= last[1] and now[1] >= now[0], n
        last = now


@pytest.mark.parametrize("most", [40, 129, 200, 256, 300, 513])
@pytest.mark.parametrize("V,D", [(5000, 264), (32000, 64)])
def test_scratch_made_for_more_rows(torch, most, V, D):
    """One buffer, made for the largest batch, serves every smaller one and calls without gradients, with the results that a buffer of the call's
    own gives; nothing behind it is touched."""
    h, w, tok, _ = inputs(torch, most, V, D, most + V)
    ctx = context(V)
    size = ctx.head_scratch(most, D, True)
    buf = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    shared, border = buf[:size], buf[size:]
    for n in [k for k in (1, 13, 40, 63, 65, 100, 128, 129, 200, 257, 512, most - 1, most) if k <= most]:
        got = []
        for sc in (shared, scratch_for(torch, ctx, n, D, True)[0]):
            rl, lp, lse = out(torch, n, 3)
            gh, gw, gh2, gw2 = [torch.full_like(t, 9.0) for t in (h[:n], w, h[:n], w)]
            ctx.head_cross_entropy(h[:n], w, tok[:n], rl, sc, grad_hidden_out=gh, grad_weight_out=gw)
            ctx.head_logprob(h[:n], w, tok[:n], lp, sc, lse_out=lse)
            ctx.head_logprob_grad(h[:n], w, tok[:n], lse, torch.linspace(-1.0, 1.0, n, device="cuda"), sc, grad_hidden_out=gh2, grad_weight_out=gw2)
            got.append((rl, lp, lse, gh, gw, gh2, gw2))
        assert all(torch.equal(a, b) for a, b in zip(*got)), n
        Head(h[:n], w, tok[:n]).close_logp(got[0][1])
    assert bool((border == 255).all()) and ctx.status() == 0


# ---- overlaps --------------------------------------------------------------------------------------

def test_overlaps_with_the_weight(torch):
    import paper_2512_11280_b200 as adasd
    n, V, D = 10, 300, 64
    h, w, tok, _ = inputs(torch, n, V, D, 3)
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, lp, total = out(torch, n, 2) + out(torch, 1)
    inside = w.view(-1).view(torch.float32)                  # the weight's memory as fp32
    for bad in (dict(grad_hidden_out=w[:n]), dict(grad_weight_out=w), dict(logp_out=inside[5:5 + n]), dict(loss_out=inside[-1:]), dict(logp_out=rl),
                dict(lse_out=sc[:4 * n].view(torch.float32)), dict(row_weight=rl), dict(row_weight=sc[:4 * n].view(torch.float32))):
        before = w.clone()
        with pytest.raises(adasd.AdasdError) as err:
            ctx.head_cross_entropy(h, w, tok, rl, sc, **bad)
        assert err.value.code == adasd.ERR_SHAPE, bad.keys()
        assert torch.equal(before, w)
    ctx.head_cross_entropy(h, w, tok, rl, sc, loss_out=total, logp_out=lp)
    assert ctx.status() == 0


@pytest.mark.parametrize("n,pad", [(5, 0), (100, 8), (300, 0), (300, 3)])
def test_gradients_as_columns_beside_what_they_are_of(torch, n, pad):
    """Hidden states and their gradient, weight and its gradient, side by side in one array each (pad: columns between the first two)."""
    V, D = 700, 136
    h, w, tok, _ = inputs(torch, n, V, D, n)
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, rl2 = out(torch, n, 2)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    ctx.head_cross_entropy(h, w, tok, rl, sc, grad_hidden_out=gh, grad_weight_out=gw)
    hb, wb = torch.full((n, 2 * D + pad), 9.0, device="cuda").bfloat16(), torch.full((V, 2 * D), 9.0, device="cuda").bfloat16()
    hb[:, :D], wb[:, D:] = h, w
    ctx.head_cross_entropy(hb[:, :D], wb[:, D:], tok, rl2, sc, grad_hidden_out=hb[:, D + pad:], grad_weight_out=wb[:, :D])
    assert torch.equal(rl, rl2) and torch.equal(hb[:, D + pad:], gh) and torch.equal(wb[:, :D], gw)
    assert torch.equal(hb[:, :D], h) and torch.equal(wb[:, D:], w) and bool((hb[:, D:D + pad] == 9.0).all())
    assert ctx.status() == 0


# ---- confident rows --------------------------------------------------------------------------------

@pytest.mark.parametrize("n,offset", [(7, 0), (7, 1), (100, 0), (200, 0)])
def test_confident_rows_of_large_logits(torch, n, offset):
    """Logits of 64 to 519 whose token has 1 - p = 7e-5.  h = (a, 1, 0 ..), w = (1, 0 ..) and at the token (1, 11.5, 0 ..): z is exact, grad_h has the sum of the row's
    G = dL/dz, which is 0, in column 0, and 11.5 (p - 1) in column 1.  S = 1 + 7e-5 comes from 2^t of the token (2^-22 of itself) and 5 additions, 2^-24 each:
    p - 1 is off by 9 * 2^-24 for all of it, where lse in 32 bits would take 2^-24 of 519 and more.  The other columns' p, 1e-5 each, add nothing to that."""
    V, D, U = 8, 8, 2.0 ** -24
    h = torch.zeros(n * D + offset, device="cuda").bfloat16()[offset:].view(n, D)
    a = (torch.linspace(64.0, 508.0, n, device="cuda") + 0.37).bfloat16()
    h[:, 0], h[:, 1] = a, 1.0
    w = torch.zeros(V, D, device="cuda").bfloat16()
    w[:, 0], w[3, 1] = 1.0, 11.5
    tok = torch.full((n,), 3, dtype=torch.int32, device="cuda")
    z = (h.double() @ w.double().t())
    p1 = torch.expm1(torch.log_softmax(z, -1)[:, 3])         # (z - a is exact: 0 and 11.5)
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, lp, lse = out(torch, n, 3)
    gh = torch.full((n, D), 9.0, device="cuda").bfloat16()
    ctx.head_cross_entropy(h, w, tok, rl, sc, grad_hidden_out=gh)
    assert bool((gh[:, 0].double().abs() <= 10 * U).all()), float(gh[:, 0].double().abs().max() / U)
    assert bool(((gh[:, 1].double() - 11.5 * p1).abs() <= 11.5 * 10 * U + 2.0 ** -8 * 11.5 * p1.abs()).all())
    assert bool((gh[:, 1] < 0).all()) and bool((gh[:, 2:] == 0).all())
    # from an lse in 32 bits p - 1 is off by as much as that is, but p is not above 1
    ctx.head_logprob(h, w, tok, lp, sc, lse_out=lse)
    ctx.head_logprob_grad(h, w, tok, lse, torch.ones(n, device="cuda"), sc, grad_hidden_out=gh)
    assert bool((gh[:, 1] >= 0).all()), float(gh[:, 1].min())
    assert ctx.status() == 0


# ---- logits that are not finite though the given lse is --------------------------------------------

@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("n", [6, 60, 100, 200])
@pytest.mark.parametrize("which", ["hidden", "weight", "both"])
def test_logits_that_are_not_finite_with_a_finite_lse(torch, n, value, which):
    """The weight changed between the forward pass and the backward pass: a row of it is not finite now."""
    import paper_2512_11280_b200 as adasd
    V, D = 900, 64
    h, w, tok, _ = inputs(torch, n, V, D, 8)
    h[:, 5] = 1.0
    tok[0], tok[4] = 7, -1
    on = (tok >= 0) & (tok < V)
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    lp, H, lse = out(torch, n, 3)
    ctx.head_logprob(h, w, tok, lp, sc, H, lse)
    dl, dH = torch.linspace(0.5, 1.0, n, device="cuda"), torch.linspace(-1.0, -0.5, n, device="cuda")
    for ent in (None, H):
        for broken in (False, True):
            w2 = w.clone()
            if broken:
                w2[333, 5] = value
            gh, gw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
            ctx.head_logprob_grad(h, w2, tok, lse, dl, sc, entropy=ent, grad_entropy=None if ent is None else dH,
                                  grad_hidden_out=None if which == "weight" else gh, grad_weight_out=None if which == "hidden" else gw)
            assert ctx.status() == (adasd.STATUS_NAN if broken else 0)
            if which != "weight":
                assert bool((torch.isfinite(gh[on]).all(-1) != broken).all()) and bool((gh[~on] == 0).all())
            if which != "hidden":
                fine = torch.isfinite(gw).all(-1)
                assert bool(fine[333]) != broken and int(fine.sum()) == (V - 1 if broken else V)
    # nobody's row: none is looked at
    w[333, 5] = value
    ctx.head_logprob_grad(h, w, torch.full_like(tok, -1), lse, dl, sc, grad_hidden_out=gh, grad_weight_out=gw)
    assert ctx.status() == 0 and bool((gh == 0).all()) and bool((gw == 0).all())


# ---- long sums -------------------------------------------------------------------------------------

@pytest.mark.parametrize("n,masked", [(32768, 0.0), (32769, 0.0), (32833, 0.0), (65537, 0.0), (100001, 0.3), (140001, 0.9)])
def test_rows_about_the_parts_of_the_weight_gradients_sums(torch, n, masked):
    V, D = 300, 72
    h, w, tok, g = inputs(torch, n, V, D, n, out=masked)
    ctx, ref = context(V), Head(h, w, tok)
    sc, border = scratch_for(torch, ctx, n, D, True)
    rl, total = out(torch, n) + out(torch, 1)
    gh, gw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
    ctx.head_cross_entropy(h, w, tok, rl, sc, scale=1.0 / n, loss_out=total, grad_hidden_out=gh, grad_weight_out=gw)
    loss, tol, G, size = ref.cross_entropy(None, 0.0, 0.0, 1.0 / n)
    assert bool(((rl.double() - loss).abs() <= tol).all())
    assert abs(float(total) - float(loss.sum())) <= float(tol.sum()) + 2.0 ** -24 * abs(float(loss.sum()))
    ref.close_grads(G, size, gh, gw)
    assert bool((border == 255).all()) and ctx.status() == 0


def test_sums_over_many_rows_are_not_cut(torch):
    """grad_w of 2^20 rows, every product of a sum of one sign.  A product is cut where it is lined up with the accumulator, 25 places below its first: half of 2^-25 of the
    sum so far, in the mean half of the whole; the sum of 16 products is cut again at 2^-23.  2^-27 + 2^-25 / 16 for every product, at the most, are 3.1e-4 of a part of 2^15
    products (and 1e-2 of all in one sum).  Roundings to bf16, 2^-9 / sqrt(3) in the mean square and independent (the columns have scales of their own), leave 3e-5
    of the mean over 1500 elements."""
    n, V, D = (1 << 20) + 3, 24, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    h = (torch.randn(n, D, generator=g, device="cuda").abs() * torch.exp2(torch.rand(D, generator=g, device="cuda"))).bfloat16()
    w = (torch.randn(V, D, generator=g, device="cuda") / D).bfloat16()
    tok = torch.zeros(n, dtype=torch.int32, device="cuda")
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, = out(torch, n)
    gw = torch.full_like(w, 9.0)
    ctx.head_cross_entropy(h, w, tok, rl, sc, scale=1.0 / n, grad_weight_out=gw)
    want = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for a in range(0, n, 1 << 18):
        x = h[a:a + (1 << 18)].double()
        G = torch.softmax(x @ w.double().t(), -1) / n
        G[:, 0] -= 1.0 / n
        assert bool((G[:, 0] < 0).all())
        want += G.t() @ x
    off = gw.double() / want - 1.0
    assert abs(float(off.mean())) <= 3.5e-4, float(off.mean())
    assert bool((off.abs() <= 2.0 ** -8 + 1e-3).all()) and ctx.status() == 0


def test_sums_over_a_long_vocabulary_have_parts(torch):
    """A scratch has room for grad_hidden's sums in parts of at most 2^16 of the vocabulary: here eight, beside the piece of dL/dz."""
    n, V, D = 129, 1 << 19, 16384
    assert context(V).head_scratch(n, D, True) >= 256 * V * 2 + 8 * 256 * D * 4


# ---- what rounding takes from dL/dz ----------------------------------------------------------------

@pytest.mark.parametrize("n,V,D", [(40, 3000, 64), (70, 3000, 64), (128, 2000, 256), (129, 5000, 136), (300, 5000, 136), (20000, 20011, 72)])
@pytest.mark.parametrize("given", [False, True])
def test_weights_with_a_common_direction(torch, n, V, D, given):
    """w_v = noise - 30 u: what rounding takes from a row's G, summed, would be multiplied with 30 u, which the exact gradient has none of (a row's G adds up to 0).
    Left in, grad_h is 0.03 off; given back along another row than the token's, 0.0022.  Expected is the final rounding to bf16, 0.43 * 2^-8 in the mean square, and
    independent of that what is left of G's, the errors times w_v - w_x, worked out in 64 bits (up to 64 rows G has a second plane: nothing); a tenth more for chance."""
    g = torch.Generator(device="cuda").manual_seed(n + V)
    u = torch.randn(D, generator=g, device="cuda")
    u /= u.norm()
    w = (torch.randn(V, D, generator=g, device="cuda") / D ** 0.5 - 30.0 * u).bfloat16()
    h = torch.randn(n, D, generator=g, device="cuda")
    h = ((h - (h @ u)[:, None] * u) * 2.0 + u).bfloat16()
    rows = min(n, 300)                       # those that are looked at
    z = h[:rows].double() @ w.double().t()
    tok = torch.randint(0, V, (n,), generator=g, device="cuda").int()
    tok[:rows] = torch.multinomial(torch.softmax(z, -1), 1, generator=g)[:, 0].int()
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, lse = out(torch, n, 2)
    gh = torch.full_like(h, 9.0)
    if given:
        ctx.head_logprob(h, w, tok, rl, sc, lse_out=lse)
        ctx.head_logprob_grad(h, w, tok, lse, torch.full_like(lse, -1.0), sc, grad_hidden_out=gh)
    else:
        ctx.head_cross_entropy(h, w, tok, rl, sc, grad_hidden_out=gh)
    G = torch.softmax(z, -1).scatter_add_(1, tok[:rows].long()[:, None], torch.full((rows, 1), -1.0, dtype=torch.float64, device="cuda"))
    want = G @ w.double()
    e = G.float().bfloat16().double() - G
    left = e @ w.double() - e.sum(-1, keepdim=True) * w[tok[:rows].long()].double()
    expected = ((0.43 * 2.0 ** -8) ** 2 + (0.0 if n <= 64 else float((left.norm() / want.norm()) ** 2))) ** 0.5
    assert expected < 0.002
    off = float((gh[:rows].double() - want).norm() / want.norm())
    assert off <= 1.1 * expected, (off, expected)
    assert ctx.status() == 0


# ---- calls that reach branches of their own --------------------------------------------------------

@pytest.mark.parametrize("n", [16384, 16385, 30000])
@pytest.mark.parametrize("grad", [False, True])
def test_total_of_many_rows(torch, n, grad):
    """Up to 16384 rows the last row's CTA adds the losses up, beyond that a launch of its own."""
    V, D = 130, 64
    h, w, tok, g = inputs(torch, n, V, D, n, out=0.2)
    weight = torch.rand(n, generator=g, device="cuda")
    ctx, ref = context(V), Head(h, w, tok, 1.0, weight)
    sc, border = scratch_for(torch, ctx, n, D, grad)
    rl, total = out(torch, n) + out(torch, 1)
    more = dict(grad_hidden_out=torch.empty_like(h), grad_weight_out=torch.empty_like(w)) if grad else {}
    for _ in range(2):
        ctx.head_cross_entropy(h, w, tok, rl, sc, row_weight=weight, z_loss=1e-3, scale=1.0 / n, loss_out=total, **more)
        loss, tol, G, size = ref.cross_entropy(weight, 0.0, 1e-3, 1.0 / n)
        assert bool(((rl.double() - loss).abs() <= tol).all())
        # (added in 64 bits, rounded once)
        assert abs(float(total) - float(rl.double().sum())) <= 2.0 ** -24 * float(rl.double().sum().abs())
    if grad:
        ref.close_grads(G, size, more["grad_hidden_out"], more["grad_weight_out"])
    assert bool((border == 255).all()) and ctx.status() == 0


@pytest.mark.parametrize("n", [2, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("which", ["hidden", "weight", "both"])
def test_entropy_gradients_of_few_rows(torch, n, offset, which):
    """Rows as they lie (offset 0) and put together first; dL/dH alone for one of them."""
    V, D = 1100, 136
    hv, w, tok, g = inputs(torch, n, V, D, n, out=0.2)
    h = torch.empty(n * D + offset, dtype=torch.bfloat16, device="cuda")[offset:].view(n, D)
    h.copy_(hv)
    ctx, ref = context(V, 0.9), Head(h, w, tok, 0.9)
    sc, border = scratch_for(torch, ctx, n, D, True)
    lp, H, lse = out(torch, n, 3)
    ctx.head_logprob(h, w, tok, lp, sc, H, lse)
    ref.close_H(H)
    dl, dH = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    dl[0] = 0.0
    gh, gw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
    ctx.head_logprob_grad(h, w, tok, lse, dl, sc, entropy=H, grad_entropy=dH, grad_hidden_out=None if which == "weight" else gh,
                          grad_weight_out=None if which == "hidden" else gw)
    G, size = ref.given(dl, dH)
    ref.close_grads(G, size, None if which == "weight" else gh, None if which == "hidden" else gw)
    assert bool((border == 255).all()) and ctx.status() == 0


@pytest.mark.parametrize("n,D", [(128, 512), (128, 4096), (4096, 512), (4096, 4096)])
@pytest.mark.parametrize("kind", ["positive", "few large", "few alone", "log-normal", "large first", "large last"])
def test_logits_of_channels_of_very_different_size(torch, n, D, kind):
    """With a vocabulary of one token lse is the logit.  What the accumulator cuts off hangs on how a sum grows, what is put back is the mean for independent products, 3.9e-7 of
    the logit at the most (and 2^-24 of the constant's own rounding): where few products make the sum, nothing or 31 times (a part's steps after the first) half of 2^-23 of it is cut, 1.85e-6.  Regression of the errors
    on the logits; the largest, where the large products come first, was -6.3e-7."""
    g = torch.Generator(device="cuda").manual_seed(n + D)
    h, w = torch.randn(n, D, generator=g, device="cuda"), torch.randn(1, D, generator=g, device="cuda")
    few = torch.randperm(D, generator=g, device="cuda")[:4]
    scale = torch.ones(D, device="cuda")
    if kind == "positive":
        h, w = h.abs(), w.abs()
    elif kind == "few large":
        scale[few] = 300.0
    elif kind == "few alone":
        scale.zero_()[few] = 300.0
    elif kind == "log-normal":
        scale = torch.exp(2 * torch.randn(D, generator=g, device="cuda"))
    else:
        scale[slice(0, 4) if kind == "large first" else slice(-4, None)] = 3000.0
    h, w = (h * scale).bfloat16(), w.bfloat16()
    ctx = context(1)
    sc, _ = scratch_for(torch, ctx, n, D, False)
    lp, lse = out(torch, n, 2)
    ctx.head_logprob(h, w, torch.zeros(n, dtype=torch.int32, device="cuda"), lp, sc, lse_out=lse)
    z, size = (h.double() @ w.double().t())[:, 0], (h.double().abs() @ w.double().abs().t())[:, 0]
    off = lse.double() - z
    assert -1.85e-6 <= float((off * z).sum() / (z * z).sum()) <= 3.9e-7 + 2.0 ** -24
    assert bool((off.abs() <= (D / 16 + 2) * 2.0 ** -23 * size).all()) and ctx.status() == 0


# ---- several at once -------------------------------------------------------------------------------

def test_many_rows_captured_beside_few_on_another_stream(torch):
    """One graph of a call whose sums come in parts, replayed with other masks, while calls of few rows run on a stream of their own: the results are those of each alone."""
    n, V, D = 40000, 300, 64
    ctx = context(V)
    h, w, tok, g = inputs(torch, n, V, D, 31, out=0.1)
    few = inputs(torch, 60, V, D, 32)
    big, small = scratch_for(torch, ctx, n, D, True)[0], scratch_for(torch, ctx, 60, D, True)[0]
    rl, total, gh, gw = out(torch, n) + out(torch, 1) + [torch.empty_like(h), torch.empty_like(w)]
    rl2, gh2, gw2 = out(torch, 60) + [torch.empty_like(few[0]), torch.empty_like(w)]

    def many():
        ctx.head_cross_entropy(h, w, tok, rl, big, loss_out=total, grad_hidden_out=gh, grad_weight_out=gw)

    def short():
        ctx.head_cross_entropy(few[0], few[1], few[2], rl2, small, grad_hidden_out=gh2, grad_weight_out=gw2)
    short()
    want2 = [t.clone() for t in (rl2, gh2, gw2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        many()
    side = torch.cuda.Stream()
    for share in (0.1, 1.0, 0.5, 0.0):
        tok.copy_(inputs(torch, n, V, D, 40 + int(10 * share), out=share)[2])
        many()
        want = [t.clone() for t in (rl, total, gh, gw)]
        Head(h[:4000], w, tok[:4000]).close_logp(-rl[:4000])
        for t in (rl, total, gh, gw, rl2, gh2, gw2):
            t.fill_(9.0)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            short()
        graph.replay()
        with torch.cuda.stream(side):
            short()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(want + want2, (rl, total, gh, gw, rl2, gh2, gw2))), share
    assert ctx.status() == 0
