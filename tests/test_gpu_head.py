"""Log-probs, cross entropy and gradients straight from hidden states, against 64 bits."""
import pytest

from tests.head_reference import H16, U, Head

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return torch


_ctx = {}


def context(V, T=1.0):
    import paper_2512_11280_b200 as adasd
    if V not in _ctx:
        _ctx[V] = adasd.Context(1, V, 1, list_capacity=1)
    _ctx[V].set_warpers(T)
    return _ctx[V]


def inputs(torch, n, V, D, seed, scale=2.0, out=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(n, D, generator=g, device="cuda").bfloat16()
    w = (torch.randn(V, D, generator=g, device="cuda") * (scale / D ** 0.5)).bfloat16()
    tok = torch.randint(0, V, (n,), generator=g, device="cuda").int()
    if n > 3:
        tok[torch.rand(n, generator=g, device="cuda") < out] = -100
        tok[1], tok[2] = V, 2 ** 31 - 1
    return h, w, tok, g


def scratch_for(torch, ctx, n, D, grad):
    """Exactly what is asked for, full of NaN, with a border that must stay."""
    size = ctx.head_scratch(n, D, grad)
    buf = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    return buf[:size], buf[size:]


def out(torch, n, k=1):
    return [torch.full((n,), -7.0, device="cuda") for _ in range(k)]


SIZES = [(1, 1, 8), (1, 5, 8), (3, 255, 16), (2, 256, 64), (5, 257, 72), (7, 1000, 200), (128, 300, 64), (129, 513, 136), (200, 5000, 520),
         (300, 32000, 128), (1, 32000, 2048), (64, 128256, 256), (1000, 2001, 64), (17, 70001, 1000), (600, 3001, 4096)]


@pytest.mark.parametrize("n,V,D", SIZES)
def test_logprob(torch, n, V, D):
    h, w, tok, _ = inputs(torch, n, V, D, n + V + D)
    for T in (1.0, 0.7):
        ctx, ref = context(V, T), Head(h, w, tok, T)
        sc, border = scratch_for(torch, ctx, n, D, False)
        lp, H, lse = out(torch, n, 3)
        ctx.head_logprob(h, w, tok, lp, sc, H, lse)
        ref.close_logp(lp)
        ref.close_lse(lse)
        ref.close_H(H)
        only, = out(torch, n)
        ctx.head_logprob(h, w, tok, only, sc)
        assert torch.equal(only, lp)
        assert bool((border == 255).all()) and ctx.status() == 0


@pytest.mark.parametrize("n,V,D", SIZES)
def test_cross_entropy_and_gradients(torch, n, V, D):
    h, w, tok, g = inputs(torch, n, V, D, 3 * n + V + D)
    weight = torch.rand(n, generator=g, device="cuda") + 0.5
    if n > 4:
        weight[4] = 0.0
    for e, c, T in ((0.0, 0.0, 1.0), (0.1, 1e-3, 1.3)):
        ctx, ref = context(V, T), Head(h, w, tok, T, weight)
        loss, tol, G, size = ref.cross_entropy(weight, e, c, 0.25)
        sc, border = scratch_for(torch, ctx, n, D, True)
        rl, lp, lse, total = out(torch, n, 3) + out(torch, 1)
        gh, gw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
        ctx.head_cross_entropy(h, w, tok, rl, sc, row_weight=weight, label_smoothing=e, z_loss=c, scale=0.25, loss_out=total, logp_out=lp, lse_out=lse,
                               grad_hidden_out=gh, grad_weight_out=gw)
        ref.close_logp(lp)
        ref.close_lse(lse)
        d = (rl.double() - loss).abs()
        assert bool((d <= tol).all()), float((d / tol.clamp(min=1e-30)).max())
        assert abs(float(total) - float(loss.sum())) <= float(tol.sum()) + U * abs(float(loss.sum()))
        ref.close_grads(G, size, gh, gw)
        assert bool((gh[~ref.on] == 0).all())
        # the loss alone, and either gradient alone, are the same values
        rl2, = out(torch, n)
        ctx.head_cross_entropy(h, w, tok, rl2, sc, row_weight=weight, label_smoothing=e, z_loss=c, scale=0.25)
        assert torch.equal(rl, rl2)
        gh2, gw2 = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
        ctx.head_cross_entropy(h, w, tok, rl2, sc, row_weight=weight, label_smoothing=e, z_loss=c, scale=0.25, grad_hidden_out=gh2)
        ctx.head_cross_entropy(h, w, tok, rl2, sc, row_weight=weight, label_smoothing=e, z_loss=c, scale=0.25, grad_weight_out=gw2)
        assert torch.equal(gh, gh2) and torch.equal(gw, gw2)
        assert bool((border == 255).all()) and ctx.status() == 0


@pytest.mark.parametrize("n,V,D", [(1, 40, 8), (9, 257, 72), (130, 1500, 128), (300, 32000, 256)])
@pytest.mark.parametrize("entropy", [False, True])
def test_logprob_gradient(torch, n, V, D, entropy):
    h, w, tok, g = inputs(torch, n, V, D, n + V)
    for T in (1.0, 0.8):
        ctx, ref = context(V, T), Head(h, w, tok, T)
        sc, _ = scratch_for(torch, ctx, n, D, True)
        lp, H, lse = out(torch, n, 3)
        ctx.head_logprob(h, w, tok, lp, sc, H, lse)
        dl = torch.randn(n, generator=g, device="cuda")
        dH = torch.randn(n, generator=g, device="cuda") if entropy else None
        if n > 8:
            dl[7] = 0.0                      # left out unless its entropy counts
        gh, gw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
        ctx.head_logprob_grad(h, w, tok, lse, dl, sc, entropy=H if entropy else None, grad_entropy=dH, grad_hidden_out=gh, grad_weight_out=gw)
        G, size = ref.given(dl, dH)
        ref.close_grads(G, size, gh, gw)
        assert ctx.status() == 0


# rows about 16 (what the products along few rows take at a time), a plane of 64 and a tile of 128; a vocabulary of more than one piece for few rows
@pytest.mark.parametrize("n,V,D", [(15, 400, 64), (16, 400, 136), (17, 3000, 64), (63, 500, 72), (64, 777, 256), (65, 700, 136), (112, 1500, 64), (127, 257, 520),
                                   (128, 900, 1032), (129, 255, 72), (256, 600, 200), (257, 513, 64), (3, 1050000, 8), (100, 1049000, 8)])
def test_few_rows(torch, n, V, D):
    h, w, tok, g = inputs(torch, n, V, D, n + V, out=0.3)
    ctx, ref = context(V), Head(h, w, tok)
    sc, border = scratch_for(torch, ctx, n, D, True)
    rl, lp, lse, H, total = out(torch, n, 4) + out(torch, 1)
    gh, gw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
    ctx.head_cross_entropy(h, w, tok, rl, sc, label_smoothing=0.05, scale=0.5, loss_out=total, logp_out=lp, grad_hidden_out=gh, grad_weight_out=gw)
    loss, tol, G, size = ref.cross_entropy(None, 0.05, 0.0, 0.5)
    assert bool(((rl.double() - loss).abs() <= tol).all())
    assert abs(float(total) - float(rl.double().sum())) <= 2 * U * float(rl.double().abs().sum())
    ref.close_logp(lp)
    ref.close_grads(G, size, gh, gw)
    # by given dL/dl, from a forward pass in a scratch of its own size
    sc2, border2 = scratch_for(torch, ctx, n, D, False)
    ctx.head_logprob(h, w, tok, lp, sc2, H, lse)
    ref.close_logp(lp)
    ref.close_lse(lse)
    dl = torch.randn(n, generator=g, device="cuda")
    gh.fill_(9.0)
    gw.fill_(9.0)
    ctx.head_logprob_grad(h, w, tok, lse, dl, sc, grad_hidden_out=gh, grad_weight_out=gw)
    G, size = ref.given(dl, None)
    ref.close_grads(G, size, gh, gw)
    assert bool((border == 255).all()) and bool((border2 == 255).all()) and ctx.status() == 0


@pytest.mark.parametrize("n", [129, 144, 145, 161, 200, 255, 257, 287, 288, 289])
@pytest.mark.parametrize("D", [8, 256, 264, 520, 1032])
def test_rows_of_a_round(torch, n, D):
    """Rows about one and two tiles of a pair, the last one nearly empty; dims of 1, 4, 5, 9 and 17 steps (sums come in parts of 8)."""
    for V in (31, 700, 40001):
        h, w, tok, g = inputs(torch, n, V, D, n + V + D, out=0.2)
        weight = torch.rand(n, generator=g, device="cuda") + 0.5
        ctx, ref = context(V, 0.9), Head(h, w, tok, 0.9, weight)
        sc, border = scratch_for(torch, ctx, n, D, False)
        rl, lp, lse, H = out(torch, n, 4)
        ctx.head_cross_entropy(h, w, tok, rl, sc, row_weight=weight, label_smoothing=0.1, z_loss=1e-3, logp_out=lp, lse_out=lse)
        loss, tol, _, _ = ref.cross_entropy(weight, 0.1, 1e-3, 1.0)
        assert bool(((rl.double() - loss).abs() <= tol).all())
        ref.close_logp(lp)
        ref.close_lse(lse)
        ref = Head(h, w, tok, 0.9)
        ctx.head_logprob(h, w, tok, lp, sc, H, lse)
        ref.close_logp(lp)
        ref.close_H(H)
        assert bool((border == 255).all()) and ctx.status() == 0


@pytest.mark.parametrize("n,D", [(4096, 4096), (4096, 520), (128, 4096)])
def test_logits_lose_nothing_in_the_mean(torch, n, D):
    """With a vocabulary of one token lse is the logit.  The accumulator is cut with every 16 products; of 4096 logits the errors' regression on the
    logits is within 1e-7 (it was 3.9e-7 with 512 products to a part; their own spread, 2.5e-7 of the size, leaves 4e-9 of 4096 logits and 2.2e-8 of 128)."""
    g = torch.Generator(device="cuda").manual_seed(n + D)
    h, w = torch.randn(n, D, generator=g, device="cuda").bfloat16(), torch.randn(1, D, generator=g, device="cuda").bfloat16()
    ctx = context(1)
    sc, _ = scratch_for(torch, ctx, n, D, False)
    lp, lse = out(torch, n, 2)
    ctx.head_logprob(h, w, torch.zeros(n, dtype=torch.int32, device="cuda"), lp, sc, lse_out=lse)
    z = (h.double() @ w.double().t())[:, 0]
    assert abs(float(((lse.double() - z) * z).sum() / (z * z).sum())) < 1e-7
    assert float((lse.double() - z).norm() / z.norm()) < 5e-7 and bool((lp.abs() < 1e-5).all())


def test_captured_ahead_of_any_other_call(torch):
    """In a process of its own: the first calls of all are captured."""
    import os
    import subprocess
    import sys
    code = """
import torch, paper_2512_11280_b200 as adasd
torch.manual_seed(0)
for n in (5, 200):
    V, D = 1000, 64
    h, w = torch.randn(n, D, device="cuda").bfloat16(), (torch.randn(V, D, device="cuda") / 8).bfloat16()
    tok = torch.randint(0, V, (n,), device="cuda").int()
    ctx = adasd.Context(1, V, 1, list_capacity=1)
    sc = torch.empty(ctx.head_scratch(n, D, True), dtype=torch.uint8, device="cuda")
    t = dict(param=w.float(), param_copy=w, grad=torch.empty_like(w), exp_avg=torch.zeros(V, D, device="cuda"), exp_avg_sq=torch.zeros(V, D, device="cuda"))
    rl, gh = torch.empty(n, device="cuda"), torch.empty_like(h)
    table = ctx.adamw_table([t])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.head_cross_entropy(h, w, tok, rl, sc, scale=1.0 / n, grad_hidden_out=gh, grad_weight_out=t["grad"])
        ctx.adamw_step(table, 1e-2, 1)
    ref = -torch.log_softmax(h.double() @ w.double().t(), -1).gather(1, tok.long()[:, None])[:, 0] / n
    g.replay()
    torch.cuda.synchronize()
    assert float((rl - ref).abs().max()) < 1e-4, float((rl - ref).abs().max())
    assert bool((w == t["param"].bfloat16()).all()) and bool(t["grad"].any()) and ctx.status() == 0
print("fine")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("n,V,D", [(70000, 5000, 64), (20000, 20011, 72)])
def test_vocabulary_in_pieces(torch, n, V, D):
    """So many rows that the gradient's piece holds a part of the vocabulary; checked on parts of rows."""
    h, w, tok, g = inputs(torch, n, V, D, 11, out=0.3)
    ctx = context(V)
    sc, border = scratch_for(torch, ctx, n, D, True)
    rl, = out(torch, n)
    gh, gw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
    ctx.head_cross_entropy(h, w, tok, rl, sc, scale=1.0 / n, grad_hidden_out=gh, grad_weight_out=gw)
    assert bool((border == 255).all())
    want_w = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    tol_w, terms = want_w.clone(), want_w.clone()
    for a in range(0, n, 4000):
        ref = Head(h[a:a + 4000], w, tok[a:a + 4000])
        loss, tol, G, size = ref.cross_entropy(None, 0.0, 0.0, 1.0 / n)
        assert bool(((rl[a:a + 4000].double() - loss).abs() <= tol).all())
        ref.close_grads(G, size, gh[a:a + 4000], None)
        dG = H16 * G.abs() + (1 + H16) * (ref.el + 2 * U * ref.lnp.abs().amax(-1))[:, None] * size
        want_w += G.t() @ ref.h
        tol_w += dG.t() @ ref.h.abs()
        terms += G.abs().t() @ ref.h.abs()
    tol_w += (n / 8 + 68) * U * terms
    d = (gw.double() - want_w).abs()
    assert bool((d <= tol_w * (1 + H16) + H16 * want_w.abs()).all())
    assert float(d.norm()) <= H16 * float(want_w.norm())
    assert ctx.status() == 0


def strided(torch, values, offset, pad, fill=7.0):
    n, D = values.shape
    buf = torch.full((offset + n * (D + pad) + 64,), fill, dtype=values.dtype, device="cuda")
    view = buf[offset:offset + n * (D + pad)].view(n, D + pad)[:, :D]
    view.copy_(values)
    return view, buf


@pytest.mark.parametrize("hs,ws,ghs,gws", [((0, 0), (0, 8), (0, 0), (0, 0)), ((1, 0), (8, 0), (3, 5), (8, 8)), ((3, 5), (0, 0), (0, 8), (0, 16)),
                                           ((8, 8), (16, 24), (1, 1), (0, 0))])
@pytest.mark.parametrize("n,V,D", [(5, 300, 72), (140, 1000, 320)])
def test_strides_and_offsets(torch, n, V, D, hs, ws, ghs, gws):
    """Offsets and gaps (elements) of hidden states, weight and gradients; what lies between the rows stays and is not read."""
    hv, wv, tok, _ = inputs(torch, n, V, D, 5)
    h, hb = strided(torch, hv, *hs, fill=float("nan"))
    w, wb = strided(torch, wv, *ws, fill=float("nan"))
    gh, ghb = strided(torch, torch.zeros_like(hv), *ghs)
    gw, gwb = strided(torch, torch.zeros_like(wv), *gws)
    gh.fill_(9.0)
    gw.fill_(9.0)
    ctx, ref = context(V), Head(hv, wv, tok)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, = out(torch, n)
    ctx.head_cross_entropy(h, w, tok, rl, sc, grad_hidden_out=gh, grad_weight_out=gw)
    loss, tol, G, size = ref.cross_entropy(None, 0.0, 0.0, 1.0)
    assert bool(((rl.double() - loss).abs() <= tol).all())
    ref.close_grads(G, size, gh, gw)
    for view, buf, (offset, pad) in ((gh, ghb, ghs), (gw, gwb, gws)):
        rows, width = view.shape
        inside = torch.zeros_like(buf, dtype=torch.bool)
        inside[offset:offset + rows * (width + pad)].view(rows, width + pad)[:, :width] = True
        assert bool((buf[~inside] == 7.0).all())
    assert ctx.status() == 0


def test_rows_left_out_may_hold_anything(torch):
    n, V, D = 300, 700, 128
    h, w, tok, g = inputs(torch, n, V, D, 6, out=0.5)
    weight = torch.rand(n, generator=g, device="cuda") + 0.1
    weight[::7] = 0.0
    ref = Head(h, w, tok, 1.0, weight)
    clean = h.clone()
    h[~ref.on] = float("nan")
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, lp, H, gh, gw = out(torch, n, 3) + [torch.full_like(h, 9.0), torch.full_like(w, 9.0)]
    ctx.head_cross_entropy(h, w, tok, rl, sc, row_weight=weight, logp_out=lp, grad_hidden_out=gh, grad_weight_out=gw)
    _, _, G, size = ref.cross_entropy(weight, 0.0, 0.0, 1.0)
    ref.close_grads(G, size, gh, gw)
    ref.close_logp(lp)
    assert bool((rl[~ref.on] == 0).all()) and bool((gh[~ref.on] == 0).all())
    # the same rows, with nothing unusual in those left out: the same values
    gh2, gw2 = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
    ctx.head_cross_entropy(clean, w, tok, rl, sc, row_weight=weight, grad_hidden_out=gh2, grad_weight_out=gw2)
    assert torch.equal(gh, gh2) and torch.equal(gw, gw2)
    assert ctx.status() == 0
    # none left
    rl.fill_(5.0)
    ctx.head_cross_entropy(h, w, torch.full_like(tok, -1), rl, sc, logp_out=lp, lse_out=H, grad_hidden_out=gh, grad_weight_out=gw)
    for t in (rl, lp, H, gh, gw):
        assert bool((t == 0).all())
    assert ctx.status() == 0


def test_no_rows(torch):
    V, D = 300, 64
    _, w, _, _ = inputs(torch, 1, V, D, 6)
    ctx = context(V)
    h, tok = torch.empty(0, D, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    e, gw, total = torch.empty(0, device="cuda"), torch.full((V, D), 9.0, device="cuda").bfloat16(), torch.ones(1, device="cuda")
    sc = torch.empty(ctx.head_scratch(0, D, True), dtype=torch.uint8, device="cuda")
    ctx.head_logprob(h, w, tok, e, sc)
    ctx.head_cross_entropy(h, w, tok, e, sc, loss_out=total, grad_hidden_out=torch.empty_like(h), grad_weight_out=gw)
    assert float(total) == 0.0 and bool((gw == 0).all())
    assert ctx.status() == 0


def test_rows_that_are_not_finite(torch):
    import paper_2512_11280_b200 as adasd
    n, V, D = 200, 900, 64
    h, w, tok, _ = inputs(torch, n, V, D, 8, out=0.0)
    tok[:] = tok.clamp(0, V - 1)
    ref = Head(h, w, tok)
    h[5, 3], h[150, 0] = float("nan"), float("inf")
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, lp, lse, total = out(torch, n, 3) + out(torch, 1)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    ctx.head_cross_entropy(h, w, tok, rl, sc, loss_out=total, logp_out=lp, lse_out=lse, grad_hidden_out=gh, grad_weight_out=gw)
    assert ctx.status() == adasd.STATUS_NAN and ctx.status() == 0
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[5] = bad[150] = True
    for t in (rl, lp, lse):
        assert torch.equal(torch.isnan(t), bad)
    assert bool(torch.isnan(gh[bad]).all()) and bool(torch.isfinite(gh[~bad]).all()) and bool(torch.isnan(gw).all()) and bool(torch.isnan(total).all())
    ref.on = ref.on & ~bad
    ref.close_logp(torch.where(bad, 0.0, lp))


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("n", [6, 200])
def test_weights_that_are_not_finite(torch, n, value):
    """One such weight makes a logit of every row -inf, inf or NaN."""
    import paper_2512_11280_b200 as adasd
    h, w, tok, _ = inputs(torch, n, 900, 64, 8, out=0.0)
    tok[:] = tok.clamp(0, 899)
    h[:, 5] = 1.0
    w[333, 5] = value
    ctx = context(900)
    sc, _ = scratch_for(torch, ctx, n, 64, False)
    lp, H, lse = out(torch, n, 3)
    ctx.head_logprob(h, w, tok, lp, sc, H, lse)
    assert ctx.status() == adasd.STATUS_NAN
    for t in (lp, H, lse):
        assert bool(torch.isnan(t).all())


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("n", [6, 100, 200])
def test_rows_left_out_of_weights_that_are_not_finite(torch, n, value):
    import paper_2512_11280_b200 as adasd
    V, D = 900, 64
    h, w, tok, g = inputs(torch, n, V, D, 8)
    tok[0], tok[3], tok[4] = 7, -1, 9
    h[:, 5] = 1.0
    w[333, 5] = value
    weight = torch.ones(n, device="cuda")
    weight[4] = 0.0
    on = (tok >= 0) & (tok < V)
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, lp, H, lse = out(torch, n, 4)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    ctx.head_cross_entropy(h, w, tok, rl, sc, row_weight=weight, grad_hidden_out=gh, grad_weight_out=gw)
    assert ctx.status() == adasd.STATUS_NAN
    counts = on & (weight != 0)
    assert bool(torch.isnan(gh[counts]).all()) and bool((gh[~counts] == 0).all()) and bool((rl[~counts] == 0).all())
    ctx.head_logprob(h, w, tok, lp, sc, H, lse)
    gh.fill_(9.0)
    ctx.head_logprob_grad(h, w, tok, lse, weight, sc, grad_hidden_out=gh, grad_weight_out=gw)
    assert ctx.status() == adasd.STATUS_NAN
    assert bool(torch.isnan(gh[counts]).all()) and bool((gh[~counts] == 0).all())


@pytest.mark.parametrize("n", [6, 200])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_logits_beyond_the_floor(torch, n, sign):
    """Finite logits of 1e36 in size: where a row has no others it counts as one that is not finite; a few at the lower end have p = 0."""
    import paper_2512_11280_b200 as adasd
    V, D = 900, 64
    h, w, tok, _ = inputs(torch, n, V, D, 8, out=0.0)
    tok[:] = tok.clamp(0, V - 1)
    h[:, 5], h[3, 5] = 0.0, 2.0 ** 60
    w[:, 5] = sign * 2.0 ** 60
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    lp, H, lse, rl = out(torch, n, 4)
    ctx.head_logprob(h, w, tok, lp, sc, H, lse)
    assert ctx.status() == adasd.STATUS_NAN and ctx.status() == 0
    bad = torch.arange(n, device="cuda") == 3
    for t in (lp, H, lse):
        assert torch.equal(torch.isnan(t), bad)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    ctx.head_cross_entropy(h, w, tok, rl, sc, lse_out=lse, grad_hidden_out=gh, grad_weight_out=gw)
    assert ctx.status() == adasd.STATUS_NAN
    assert torch.equal(torch.isnan(rl), bad) and torch.equal(torch.isnan(lse), bad) and bool(torch.isnan(gw).all())
    assert bool(torch.isnan(gh[bad]).all()) and bool(torch.isfinite(gh[~bad]).all())
    if sign > 0:
        return
    # 300 of the columns only, two whole tiles' halves among them, in every row: the sum of ln p is theirs
    h[:, 5], w[:, 5] = 2.0 ** 60, 0.0
    w[256:556, 5] = -(2.0 ** 60)
    tok[:] = tok % 256
    ctx.head_cross_entropy(h, w, tok, rl, sc, label_smoothing=0.5, logp_out=lp, lse_out=lse, grad_hidden_out=gh, grad_weight_out=gw)
    assert ctx.status() == 0
    # (those 300 are 2^120 and nothing to 24 bits: their sum is rounded 300 times at the most, the rest of the loss twice)
    want = 0.5 * 300 / V * 2.0 ** 120
    assert bool(((rl.double() - want).abs() <= want * 304 * 2.0 ** -24).all())
    assert bool(torch.isfinite(gh).all())
    kept = torch.ones(V, dtype=torch.bool, device="cuda")
    kept[256:556] = False
    small = Head(torch.where(torch.arange(D, device="cuda") == 5, 0.0, h.float()).bfloat16(), w[kept], tok)
    assert bool(((lp.double() - small.l).abs() <= small.el + 2.0 ** -24 * small.l.abs()).all())


def test_confident_rows(torch):
    """p of the token near 1: p - 1 is not lost; a token of tiny probability."""
    n, V, D = 130, 600, 64
    h, w, tok, g = inputs(torch, n, V, D, 9, out=0.0)
    tok[:] = tok.clamp(0, V - 1)
    scale = torch.linspace(0, 3, n, device="cuda")[:, None]
    h = (h.float() * 0.2 + scale * w[tok.long()].float() * D ** 0.5).bfloat16()
    tok[::5] = (tok[::5] + 1) % V
    ctx, ref = context(V), Head(h, w, tok)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, = out(torch, n)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    ctx.head_cross_entropy(h, w, tok, rl, sc, grad_hidden_out=gh, grad_weight_out=gw)
    loss, tol, G, size = ref.cross_entropy(None, 0.0, 0.0, 1.0)
    assert bool(((rl.double() - loss).abs() <= tol).all())
    ref.close_grads(G, size, gh, gw)


def test_gradient_against_differences(torch):
    """The formulas' gradient against differences of the loss in 64 bits; the device's is within its tolerance of the formulas'."""
    n, V, D = 12, 200, 32
    h, w, tok, g = inputs(torch, n, V, D, 10)
    ref = Head(h, w, tok)
    _, _, G, _ = ref.cross_entropy(None, 0.1, 1e-2, 1.0)
    for grad, which in ((G @ ref.w, 0), (G.t() @ ref.h, 1)):
        d = torch.randn(grad.shape, generator=g, device="cuda").double()
        f = [Head(h.double() + s * d if which == 0 else h, w.double() + s * d if which else w, tok).cross_entropy(None, 0.1, 1e-2, 1.0)[0].sum()
             for s in (1e-4, -1e-4)]
        assert abs(float((f[0] - f[1]) / 2e-4) - float((grad * d).sum())) < 1e-5 * float((grad * d).abs().sum())


def test_the_same_as_by_way_of_logits(torch):
    """head_logprob and its gradient against token_logprob on logits that torch made, with the policy loss's coefficients between."""
    n, V, D = 64, 5000, 256
    h, w, tok, g = inputs(torch, n, V, D, 12)
    ctx, ref = context(V), Head(h, w, tok)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    lp, H, lse = out(torch, n, 3)
    ctx.head_logprob(h, w, tok, lp, sc, H, lse)
    z = (h.float() @ w.float().t()).bfloat16()
    lp2, = out(torch, n)
    ctx.token_logprob(z, tok, lp2)
    assert float((lp - lp2).abs().max()) < 2 * H16 * float(z.float().abs().max())       # (logits rounded to bf16 there)
    A = torch.randn(n, generator=g, device="cuda")
    old = lp + 0.1 * torch.randn(n, generator=g, device="cuda")
    dl = -(torch.exp(lp - old) * A) * (tok >= 0)
    gh = torch.empty_like(h)
    ctx.head_logprob_grad(h, w, tok, lse, dl, sc, grad_hidden_out=gh)
    G, size = ref.given(dl, None)
    ref.close_grads(G, size, gh, None)


def test_training_steps_of_a_head(torch):
    """Loss, gradients and AdamW on the head's fp32 weight, whose bf16 copy the next step reads: every step's gradient is that of the weight as it
    then is, every step's weight that of AdamW on this gradient."""
    from tests import adamw_reference
    n, V, D = 96, 3000, 128
    h, w, tok, g = inputs(torch, n, V, D, 13)
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, total = out(torch, n) + out(torch, 1)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    for bits in (32, 8):
        copy = w.clone()
        t = dict(param=copy.float(), grad=gw, param_copy=copy, weight_decay=0.1)
        if bits == 32:
            t.update(exp_avg=torch.zeros(V, D, device="cuda"), exp_avg_sq=torch.zeros(V, D, device="cuda"))
        else:
            blocks = -(-V * D // 256)
            t.update(exp_avg=torch.zeros(V, D, device="cuda").to(torch.float8_e4m3fn), exp_avg_sq=torch.zeros(V, D, device="cuda").to(torch.float8_e5m2),
                     avg_scale=torch.zeros(blocks, device="cuda"), sq_scale=torch.zeros(blocks, device="cuda"))
        table = ctx.adamw_table([t])
        for step in (1, 2, 3):
            ref = Head(h, copy, tok)
            ctx.head_cross_entropy(h, copy, tok, rl, sc, scale=1.0 / n, loss_out=total, grad_hidden_out=gh, grad_weight_out=gw)
            loss, tol, G, size = ref.cross_entropy(None, 0.0, 0.0, 1.0 / n)
            ref.close_grads(G, size, gh, gw)
            flat = {k: (v.clone().view(-1) if hasattr(v, "view") else v) for k, v in t.items()}
            p, m, v, tp, tm, tv = adamw_reference.step(flat, 1e-2, step, 0.9, 0.99, 1e-8, 1.0)
            ctx.adamw_step(table, 1e-2, step, betas=(0.9, 0.99))
            assert bool(((t["param"].double().view(-1) - p).abs() <= tp).all())
            assert torch.equal(copy, t["param"].bfloat16())
        assert ctx.status() == 0


def test_two_streams_and_twice_the_same(torch):
    n, V, D = 300, 9000, 256
    h, w, tok, _ = inputs(torch, n, V, D, 14)
    ctx = context(V)
    got = []
    torch.cuda.synchronize()
    for _ in range(4):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            sc, _ = scratch_for(torch, ctx, n, D, True)
            rl, gh, gw = out(torch, n) + [torch.empty_like(h), torch.empty_like(w)]
            ctx.head_cross_entropy(h, w, tok, rl, sc, grad_hidden_out=gh, grad_weight_out=gw)
            got.append((sc, rl, gh, gw))
    torch.cuda.synchronize()
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0][1:], other[1:]))
    assert ctx.status() == 0


def test_captured_and_replayed(torch):
    """One graph, new inputs and another number of rows left out at every replay."""
    n, V, D = 260, 4000, 128
    h, w, tok, g = inputs(torch, n, V, D, 15)
    ctx = context(V)
    sc, _ = scratch_for(torch, ctx, n, D, True)
    rl, lp, gh, gw = out(torch, n, 2) + [torch.empty_like(h), torch.empty_like(w)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.head_cross_entropy(h, w, tok, rl, sc, logp_out=lp, grad_hidden_out=gh, grad_weight_out=gw)
    for k, share in enumerate((0.0, 0.7, 1.0, 0.2)):
        h2, w2, tok2, _ = inputs(torch, n, V, D, 20 + k, out=share)
        for a, b in ((h, h2), (w, w2), (tok, tok2)):
            a.copy_(b)
        graph.replay()
        ref = Head(h2, w2, tok2)
        loss, tol, G, size = ref.cross_entropy(None, 0.0, 0.0, 1.0)
        assert bool(((rl.double() - loss).abs() <= tol).all())
        ref.close_logp(lp)
        ref.close_grads(G, size, gh, gw)
    assert ctx.status() == 0


def test_refusals(torch):
    import paper_2512_11280_b200 as adasd
    n, V, D = 10, 100, 64
    h, w, tok, _ = inputs(torch, n, V, D, 16)
    ctx = context(V)
    sc = torch.empty(ctx.head_scratch(n, D, True), dtype=torch.uint8, device="cuda")
    rl, = out(torch, n)
    gh, gw = torch.empty_like(h), torch.empty_like(w)

    def refused(code, h=h, w=w, tok=tok, rl=rl, sc=sc, c=ctx, **more):
        with pytest.raises(adasd.AdasdError) as err:
            c.head_cross_entropy(h, w, tok, rl, sc, **more)
        assert err.value.code == code
    refused(adasd.ERR_DTYPE, h=h.float())
    refused(adasd.ERR_DTYPE, w=w.half())
    refused(adasd.ERR_DTYPE, tok=tok.long())
    refused(adasd.ERR_DEVICE, h=h.cpu())
    refused(adasd.ERR_SHAPE, w=w[:99])
    refused(adasd.ERR_SHAPE, h=h[:, :56])
    refused(adasd.ERR_SHAPE, h=h[:, :60].contiguous(), w=w[:, :60].contiguous())             # dim not a multiple of 8
    refused(adasd.ERR_SHAPE, h=h.t().contiguous().t())
    refused(adasd.ERR_SHAPE, w=torch.empty(V, D + 4, dtype=torch.bfloat16, device="cuda")[:, :D])
    refused(adasd.ERR_ALIGN, w=torch.empty(V * D + 8, dtype=torch.bfloat16, device="cuda")[4:V * D + 4].view(V, D))
    refused(adasd.ERR_SHAPE, grad_hidden_out=gh[:9])
    refused(adasd.ERR_SHAPE, grad_hidden_out=h)
    refused(adasd.ERR_SHAPE, grad_weight_out=w)
    refused(adasd.ERR_SHAPE, grad_hidden_out=sc[:n * D * 2].view(torch.bfloat16).view(n, D))
    refused(adasd.ERR_CAPACITY, sc=sc[:-1024], grad_weight_out=gw)
    refused(adasd.ERR_CAPACITY, sc=sc[:64])
    refused(adasd.ERR_SHAPE, label_smoothing=1.0)
    refused(adasd.ERR_SHAPE, z_loss=-1.0)
    fp32 = adasd.Context(1, V, 1, adasd.ADASD_FP32, list_capacity=1)
    refused(adasd.ERR_DTYPE, c=fp32)
    cut = adasd.Context(1, V, 1, list_capacity=1)
    cut.set_warpers(1.0, top_k=5)
    refused(adasd.ERR_DTYPE, c=cut)
    cut.set_warpers(1e-39)
    refused(adasd.ERR_SHAPE, c=cut)
    with pytest.raises(adasd.AdasdError) as err:
        ctx.head_logprob_grad(h, w, tok, rl, rl, sc)
    assert err.value.code == adasd.ERR_NULL
    with pytest.raises(adasd.AdasdError) as err:
        ctx.head_logprob_grad(h, w, tok, rl, rl, sc, grad_entropy=rl, grad_hidden_out=gh)
    assert err.value.code == adasd.ERR_NULL
