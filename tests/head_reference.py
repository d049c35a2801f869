"""Log-probs, cross entropy and gradients from hidden states in 64 bits, with the tolerances of the device's values.

Tolerances (U = 2^-24).  z: products of bf16 are exact; a tensor-core instruction adds 16 of them to the accumulator and may cut what lies beyond 24 bits of
the largest: 2 U of the sum of sizes A = sum |h w| for each of dim / 16 instructions, and as much for the 16 among themselves: Ez = (dim / 16 + 2) 2 U A.
t = z log2 e / T: constant and product, 2 U |t|.  A row's S: 32 additions in a thread, 8 parts, the tiles of a lane (V / 8192), 5 more, and 2^t itself (4 U):
Es = (32 + 8 + V / 8192 + 5 + 4 + 8) U, the 8 for the exponent's rounding t 2^t <= 0.54 and the rescaling.  l = z_x / T - lse: twice Ez / T, Es, 2 U (|z_x / T| + |lse|),
U |l|.  H = lse - sum p t: Es for either sum of their sizes.
G: p comes with the error of its exponent (2 Ez / T + 2 U (|t| + |lse|) + Es): of that size relative to p's terms; then half a step of bf16, 2^-8.
grad_h: the errors e_v of G's roundings enter as sum e_v (w_v - w_x), of size |e_v| (|w_v| + |w_x|) at most (with up to 64 rows, held in two planes, they do not enter).
A product with G adds its V (or n) terms in fp32: (K / 16 + 2) 2 U of the sum of sizes, a rounding U for each of at most 32 parts and of the pieces, half a step of bf16 at the end.
"""
import torch

U, H16 = 2.0 ** -24, 2.0 ** -8


class Head:
    def __init__(self, h, w, tok, T=1.0, weight=None):
        self.h, self.w, self.T, self.n, self.V, self.D = h.double(), w.double(), T, h.shape[0], w.shape[0], h.shape[1]
        self.on = (tok >= 0) & (tok < self.V)
        if weight is not None:
            self.on &= weight != 0
        self.h = torch.where(self.on[:, None], self.h, 0.0)
        self.x = torch.where(self.on, tok, 0).long()
        self.t = self.h @ self.w.t() / T
        self.lse = torch.logsumexp(self.t, -1)
        self.lnp = self.t - self.lse[:, None]
        self.p = torch.exp(self.lnp)
        self.l = self.lnp.gather(1, self.x[:, None])[:, 0]
        self.H = -(self.p * self.lnp).sum(-1)
        size = (self.h.abs() @ self.w.abs().t()).amax(-1)
        top = self.t.abs().amax(-1)
        self.Es = (57 + self.V / 8192) * U
        self.ez = (self.D / 16 + 2) * 2 * U * size / T + 2 * U * top          # of t
        self.el = 2 * self.ez + self.Es + 2 * U * (top + self.lse.abs())
        self.off = lambda v: torch.where(self.on, v, 0.0)

    def close_logp(self, got):
        self._close(got, self.off(self.l), self.el + U * self.l.abs())

    def close_lse(self, got):
        self._close(got, self.off(self.lse), self.el + U * self.lse.abs())

    def close_H(self, got):
        size = 1 + (self.p * self.lnp.abs()).sum(-1) + (self.lse - self.t.amax(-1)).abs()
        self._close(got, self.off(self.H), 2 * (self.el + self.Es) * size + U * self.H)

    def _close(self, got, want, tol):
        d = (got.double() - want).abs()
        assert bool((d <= torch.where(self.on, tol, 0.0)).all()), (float(d.max()), float((d / tol).max()))

    def cross_entropy(self, weight, e, c, scale):
        """Row losses, their tolerance, and G = dL/dz of every row with the size of its terms."""
        w = self.off((torch.ones_like(self.l) if weight is None else weight.double()) * scale)
        mean = self.lnp.mean(-1)
        loss = w * (-(1 - e) * self.l - e * mean + c * self.lse ** 2)
        size = w.abs() * ((1 - e) + e + 2 * c * self.lse.abs())
        tol = size * (self.el + self.Es) + w.abs() * e * self.V ** 0.5 * U * self.t.abs().amax(-1) + 4 * U * loss.abs() + 4 * U * w.abs() * (mean.abs() * e + self.l.abs() + c * self.lse ** 2)
        one = torch.zeros_like(self.p).scatter_(1, self.x[:, None], 1.0)
        a = 1 + 2 * c * self.lse[:, None]
        k = (w / self.T)[:, None]
        return loss, tol, k * (a * self.p - (1 - e) * one - e / self.V), k.abs() * (a * self.p + (1 - e) * one + e / self.V)

    def given(self, dl, dH):
        """G of a loss with given dL/dl and dL/dH, and the size of its terms."""
        dl, dH = self.off(dl.double())[:, None], self.off(torch.zeros_like(self.l) if dH is None else dH.double())[:, None]
        one = torch.zeros_like(self.p).scatter_(1, self.x[:, None], 1.0)
        g = (dl * (one - self.p) - dH * self.p * (self.lnp + self.H[:, None])) / self.T
        return g, (dl.abs() * (one + self.p) + dH.abs() * self.p * (self.lnp.abs() + self.H[:, None].abs() + 1)) / self.T

    def close_grads(self, G, size, grad_h, grad_w, parts=64):
        rel = (self.el + 2 * U * (self.lnp.abs().amax(-1) + self.H))[:, None]
        dG = H16 * G.abs() + (1 + H16) * rel * size
        for got, want, tol, terms, K in ((grad_h, G @ self.w, dG @ self.w.abs(), G.abs() @ self.w.abs(), self.V),
                                         (grad_w, G.t() @ self.h, dG.t() @ self.h.abs(), G.abs().t() @ self.h.abs(), self.n)):
            if got is None:
                continue
            if got is grad_h:
                tol = tol + H16 * G.abs().sum(-1, keepdim=True) * self.w[self.x].abs()
            tol = tol + ((K / 16 + 2) * 2 + parts) * U * (terms + tol)
            tol = tol + H16 * (want.abs() + tol)
            d = (got.double() - want).abs()
            assert bool((d <= tol).all()), (float(d.max()), float((d / tol.clamp(min=1e-300)).max()))
            # two roundings to bf16, spread evenly over a step of 2^-8 to 2^-7 of the value: 0.42 of 2^-8 each in the mean square, as
            # independent errors 0.6 of 2^-8 in all; a term that is left out shows here
            norm = float(want.norm())
            if want.numel() >= 4096 and norm > 0:
                assert float((got.double() - want).norm()) <= H16 * norm, float((got.double() - want).norm()) / norm
