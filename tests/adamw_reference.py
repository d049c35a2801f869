"""AdamW by its definition in 64 bits, the 8-bit formats in elementary torch operations, and the tolerances of the device's values.

Tolerances (U = 2^-24, a rounding of fp32).  m' = b1 m + (1 - b1) g: constants, the scaled gradient, products and the sum are rounded
once each: 4 U of the two terms' sizes.  v': one rounding more (the square, of a gradient that was rounded: two): 6 U of its (positive)
terms.  The step s = rate m' / (root sqrt(v') + eps): square root and reciprocal 2^-23 of themselves each at the most (2 U + 2 U), half of v's 6 U,
constants and products 6 U: 16 U of |s|, and rate / denominator times m's error.  p' = p keep - s: keep and the product round, the sum rounds: 4 U of |p|
and U of |s|.  A bf16 result adds half a step of its own, 2^-8 of |p'| (rounded up or down: a step, 2^-7).
"""
import torch

U = 2.0 ** -24
BLOCK, M_MAX, V_MAX = 256, 448.0, 57344.0


def values(t, n):
    """States in 64 bits."""
    m, v = t["exp_avg"].double(), t["exp_avg_sq"].double()
    if t["exp_avg"].dtype is not torch.float32:
        m = m * t["avg_scale"].double().repeat_interleave(BLOCK)[:n]
        v = v * t["sq_scale"].double().repeat_interleave(BLOCK)[:n]
    return m, v


def step(t, lr, t_step, b1, b2, eps, scale):
    """p', m', v' and the tolerances of each, from the tensors ahead of the step."""
    n = t["param"].numel()
    p, g = t["param"].double(), t["grad"].double() * scale
    m, v = values(t, n)
    tm, tv = (b1 * m).abs() + ((1 - b1) * g).abs(), b2 * v + (1 - b2) * g * g
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    rate, denom = lr / (1 - b1 ** t_step), torch.sqrt(v / (1 - b2 ** t_step)) + eps
    s = rate * m / denom
    p2 = p * (1 - lr * t.get("weight_decay", 0.0)) - s
    return p2, m, v, 17 * U * s.abs() + 4 * U * rate * tm / denom + 4 * U * p.abs(), 4 * U * tm, 6 * U * tv


def mix(x):
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def noise(n, seed, t_step, index, device):
    key = mix(seed ^ mix((t_step + 0x9E3779B9 * (index + 1)) & 0xFFFFFFFF))
    return mix((torch.arange(n, device=device) + key) & 0xFFFFFFFF)


def grid(y, bits, dropped, least):
    a = y.abs()
    big = ((a.view(torch.int32) + bits.int()) & -(1 << dropped)).view(torch.float32)
    small = torch.floor(a / least + bits.float() * 0.5 ** dropped) * least
    return torch.where(a < least * 2 ** (23 - dropped), small, big).copysign(y)


def codes(t, b1, b2, scale, h=None):
    """The 8-bit states after a step, in fp32 operations rounded one by one: codes and scales of m and v.  h: hash of each element."""
    n = t["param"].numel()
    f = lambda x: torch.tensor(x, dtype=torch.float32, device=t["param"].device)  # noqa: E731
    pad = lambda x: torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)  # noqa: E731
    g = t["grad"].float() * f(scale)
    m = t["exp_avg"].float() * t["avg_scale"].repeat_interleave(BLOCK)[:n]
    v = t["exp_avg_sq"].float() * t["sq_scale"].repeat_interleave(BLOCK)[:n]
    m = pad(m * f(b1) + g * f(1 - b1))
    v = pad(v * f(b2) + (g * g) * f(1 - b2))
    mt, vt = m.abs().amax(-1, keepdim=True), v.amax(-1, keepdim=True)
    y = m * torch.where(mt >= 2.0 ** -100, torch.full_like(mt, M_MAX) / mt, 0.0)
    q = v * torch.where(vt >= 2.0 ** -100, torch.full_like(vt, V_MAX) / vt, 0.0)
    if h is not None:
        h = pad(h)
        y, q = grid(y, h & 0xFFFFF, 20, 2.0 ** -9), grid(q, h >> 11, 21, 2.0 ** -16)
    y = y.clamp(-M_MAX, M_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
    q = q.clamp(max=V_MAX).to(torch.float8_e5m2).view(torch.uint8)
    q = torch.where((v > 0) & (q == 0), 1, q.int()).to(torch.uint8)
    return y.view(-1)[:n], q.view(-1)[:n], (mt * (1.0 / M_MAX))[:, 0], (vt * (1.0 / V_MAX))[:, 0]
