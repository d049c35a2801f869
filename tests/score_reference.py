"""Scoring and losses of given tokens in 64 bits, from their definitions, with the tolerances of the device's values.

Tolerances.  The device holds a row's S = sum 2^t in 32 bits: at most 128 additions by a thread, two accumulators, then trees
of at most 12 levels, so |dS| / S <= 80 2^-24 at the most; 2^t comes with 2^-22 and the rounding of t (t 2^t <= 0.54);
together under 100 2^-24 =: E.  l = z_x - m - ln S then is E off, plus half a step of its own size when it is written.
H = ln S - T / S: E for each of the two, relative to their sizes.  A gradient's p_v = 2^q: q up to 150 in size before p vanishes,
rounded twice: 2 x 150 x 2^-24 ln 2 = 21 x 2^-24, and E from ln S and 2^-22: under 130 x 2^-24; the coefficients dL/dl hang on
l (ratio e^(l - l_old), e^(l_ref - l)): E more.  R = 256 x 2^-24 of the sum of the terms' sizes covers all, then half a step of
the gradient's type.  Exponentials below 2^-125 are 0 on the device (2^t is flushed; S >= 1): 2^-125 of the row's coefficient
|dL/dl| / T, which the size at the row's token holds, and of |dL/dH| / T times a logarithm of 125 ln 2 + H < 200 at the most.
"""
import torch

E, R, U32 = 100 * 2.0 ** -24, 256 * 2.0 ** -24, 2.0 ** -24


def rows(z, tok, T=1.0):
    """ln p, p, l, H, lse, which rows count (float64; rows left out: zeros)."""
    V = z.shape[1]
    on = (tok >= 0) & (tok < V)
    m = z.double().amax(-1)
    y = (z.double() - m[:, None]) / T            # (of z / T itself 64 bits lose the difference at temperatures of 1e-9)
    lnS = torch.logsumexp(y, -1)
    lse = m / T + lnS
    lnp = y - lnS[:, None]
    p = torch.exp(lnp)
    l = lnp.gather(1, torch.where(on, tok, 0).long()[:, None])[:, 0]
    H = -torch.where(p > 0, p * lnp, 0.0).sum(-1)
    zero = torch.zeros_like(l)
    return lnp, p, torch.where(on, l, zero), torch.where(on, H, zero), torch.where(on, lse, zero), on


def gradient(lnp, p, H, tok, on, dl, dH, T):
    """dL/dz, and the size of its terms."""
    one = torch.zeros_like(p).scatter_(1, torch.where(on, tok, 0).long()[:, None], 1.0)
    dl, dH = dl[:, None], dH[:, None]
    lnp0 = torch.where(p > 0, lnp, torch.zeros_like(lnp))
    g = (dl * (one - p) - dH * p * (lnp0 + H[:, None])) / T
    size = (dl.abs() * (one + p) + dH.abs() * p * (lnp0.abs() + H[:, None].abs())) / T
    off = ~on[:, None]
    return g.masked_fill(off, 0.0), size.masked_fill(off, 0.0)


def close_logp(got, l, extra=0.0):
    tol = E + U32 * l.abs() + extra
    d = (got.double() - l).abs()
    assert bool((d <= tol).all()), (float(d.max()), float(tol.max()))


def close_entropy(got, H, lse_minus_m):
    """lse_minus_m: ln S."""
    tol = 2 * E * (1 + lse_minus_m.abs() + (lse_minus_m - H).abs()) + U32 * H.abs()
    d = (got.double() - H).abs()
    assert bool((d <= tol).all()), (float(d.max()), float((d / tol).max()))


def close_grad(got, g, size, rel=R):
    half = torch.finfo(got.dtype).eps / 2
    flushed = 2.0 ** -125 * 200 * (1 + size.amax(-1, keepdim=True)) if size.numel() else 0.0
    tol = rel * size + half * (g.abs() + rel * size) + flushed
    d = (got.double() - g).abs()
    worst = (d / tol).max() if d.numel() else 0
    assert bool((d <= tol).all()), (float(d.max()), float(worst))


def policy(l, H, on, adv, old, ref, w, lo, hi, kl, ent, scale):
    """row losses, e^r - r - 1, dL/dl, dL/dH, and the sizes of loss and dL/dl."""
    A = adv.double()
    w = (torch.ones_like(l) if w is None else w.double()) * scale
    on = on & (w != 0)
    w = torch.where(on, w, 0.0)
    ratio = torch.exp(l - old.double()) if old is not None else torch.ones_like(l)
    s1, s2 = ratio * A, ratio.clamp(1 - lo, 1 + hi) * A
    loss, dl = -torch.minimum(s1, s2), torch.where(s1 <= s2, -s1, 0.0)
    size, dsize = loss.abs(), dl.abs()
    k3 = torch.zeros_like(l)
    if ref is not None:
        r = ref.double() - l
        k3 = torch.expm1(r) - r
        loss, dl = loss + kl * k3, dl - kl * torch.expm1(r)
        size, dsize = size + kl * (torch.exp(r) + r.abs() + 1), dsize + kl * (torch.exp(r) + 1)
    loss, dH = loss - ent * H, torch.full_like(l, -ent)
    size = size + abs(ent) * (H.abs() + 30)
    z = torch.zeros_like(l)
    sel = lambda v: torch.where(on, v, z)  # noqa: E731
    return sel(loss * w), sel(k3), sel(dl * w), sel(dH * w), sel(size * w.abs()), sel(dsize * w.abs()), on


def preference(l, on, start, ref, pw, rule, beta, margin, smoothing, average, scale):
    """seq log-probs, pair losses, dL/dl of every row."""
    P = (len(start) - 1) // 2
    seq, count = [], []
    for s in range(2 * P):
        a, b = start[s], max(start[s], start[s + 1])
        n = int(on[a:b].sum())
        seq.append(torch.where(on[a:b], l[a:b], 0.0).sum() / (max(n, 1) if average else 1))
        count.append(max(n, 1) if average else 1)
    seq = torch.stack(seq)
    d = seq - (ref.double() if ref is not None else 0.0)
    D = (d[:P] - d[P:]).detach().requires_grad_(True)
    if rule == "sigmoid":
        ls, u = torch.nn.functional.logsigmoid, beta * D - margin
        loss = -(1 - smoothing) * ls(u) - smoothing * ls(-u)
    elif rule == "squared":
        loss = (D - margin - 1 / (2 * beta)) ** 2
    else:
        loss = torch.relu(1 - (beta * D - margin))
    w = scale * (pw.double() if pw is not None else torch.ones_like(D))
    loss = torch.where(w == 0, torch.zeros_like(D), w * loss)
    dD, = torch.autograd.grad(loss.sum(), D)
    dl = torch.zeros_like(l)
    for s in range(2 * P):
        a, b = start[s], max(start[s], start[s + 1])
        dl[a:b] = (dD[s] if s < P else -dD[s - P]) / count[s]
    return seq, loss.detach(), torch.where(on, dl, 0.0), dD
