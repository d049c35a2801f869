"""Training and scoring from hidden states: the cases that these operators are measured on, their plain form in
elementary torch operations, and their values in 64 bits.

h [rows, dim] are hidden states ahead of the output projection ("head"), w [V, dim] its weight, x the token of each row,
T the temperature; z = h w^T / T are never handed over.  l = ln softmax(z)_x, H the row's entropy.  A row whose token is negative is
left out (a prompt, padding): it counts nothing and its gradient is zeros.

  head_logprob        l, and H, of every row
  head_logprob_grad   gradients of h and w from given dL/dl and dL/dH
  head_cross_entropy  weighted cross entropy with label smoothing e and a term c lse^2; train: with the gradients of h and w
  adamw               one AdamW step over many tensors; states in 32 bits, or in 8 with a scale for every 256 elements

A case:
  op       one of the four
  rows, V, dim   rows of hidden states, vocabulary, width
  T        temperature
  masked   share of the rows that are left out
  train    with the gradients (head_cross_entropy without: the loss alone)
  entropy  head_logprob: H too; head_logprob_grad: with dL/dH
  smoothing, z_loss   e and c
  sizes    adamw: "even" (tensors of one size) or "model" (a few large ones, many small)
  tensors, elements   adamw: how many tensors, and elements in all
  param, grad         adamw: "bf16" or "fp32"
  bits     adamw: of the states
  copy     adamw: fp32 parameters with a bf16 copy that the model reads
  stochastic  adamw: 8-bit states and bf16 parameters rounded up or down by a hash of seed, step, tensor and element
"""
import functools
import math

import torch

own = False

BETA1, BETA2, EPS, LR, STEP, SEED, GRAD_SCALE = 0.9, 0.999, 1e-8, 3e-4, 1200, 77, 0.5
BLOCK, M_MAX, V_MAX, LEAST = 256, 448.0, 57344.0, 2.0 ** -100


def _head(op, rows, V, dim, T=1.0, masked=0.0, train=True, entropy=False, smoothing=0.0, z_loss=0.0, name=None):
    train = op == "head_logprob_grad" or (op == "head_cross_entropy" and train)
    c = dict(op=op, rows=rows, V=V, dim=dim, T=T, masked=masked, train=train, entropy=entropy, smoothing=smoothing, z_loss=z_loss)
    if name:
        c["name"] = name
    return c


def _adamw(sizes, tensors, elements, param="fp32", grad="fp32", bits=32, copy=False, stochastic=False, name=None):
    c = dict(op="adamw", sizes=sizes, tensors=tensors, elements=elements, param=param, grad=grad, bits=bits, copy=copy, stochastic=stochastic)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of one request whose caller asked for log-probs: latency
        _head("head_logprob", 1, 32000, 2048, entropy=True, name="head logprob one token"),
        # one verification round of an ordinary batch (B=32, K=8), its tokens scored
        _head("head_logprob", 288, 128256, 4096, entropy=True, name="head logprob round"),
        # sequences scored by a reference model ahead of training, a quarter of the rows prompts
        _head("head_logprob", 4096, 151936, 2048, masked=0.25, name="head logprob sequences"),
        # the backward pass of a loss of the user's own on one answer
        _head("head_logprob_grad", 60, 32000, 2048, T=0.8, name="head gradient answer"),
        # the same with an entropy bonus; vocabulary and width of no round size
        _head("head_logprob_grad", 1000, 50257, 1000, entropy=True, name="head gradient odd"),
        # one short sequence of a small draft model
        _head("head_cross_entropy", 7, 32000, 512, name="cross entropy short"),
        # a micro-batch of ordinary length, label smoothing, a tenth of the rows left out
        _head("head_cross_entropy", 2048, 128256, 2048, masked=0.1, smoothing=0.1, name="cross entropy micro-batch"),
        # the largest: long packed sequences, a quarter of the rows prompts, lse^2 term
        _head("head_cross_entropy", 8192, 151936, 4096, masked=0.25, z_loss=1e-4, name="cross entropy packed"),
        # the loss alone, as an evaluation reports it
        _head("head_cross_entropy", 999, 128256, 2048, train=False, name="cross entropy evaluation"),
        # norms and biases of a small draft model: latency
        _adamw("even", 12, 12 * 2048, name="adamw small tensors"),
        # a head's fp32 weight and the bf16 copy that the model reads
        _adamw("even", 1, 128256 * 2048, grad="bf16", copy=True, name="adamw head 32 bits"),
        # a draft model's tensors in bf16, states in 8 bits
        _adamw("model", 150, 300_000_000, param="bf16", grad="bf16", bits=8, stochastic=True, name="adamw model 8 bits"),
    ]


def draw(rng):
    def log_uniform(a, b):
        return math.exp(rng.uniform(math.log(a), math.log(b)))
    op = rng.choice(["head_logprob", "head_logprob_grad", "head_cross_entropy", "head_cross_entropy", "adamw", "adamw"])
    if op == "adamw":
        tensors = int(log_uniform(1, 400))
        bits = rng.choice([32, 8])
        param = rng.choice(["fp32", "bf16"])
        return _adamw(rng.choice(["even", "model"]), tensors, tensors + int(log_uniform(1000, 2.5e8)), param, rng.choice(["fp32", "bf16"]),
                      bits, param == "fp32" and rng.random() < 0.5, rng.random() < 0.5)
    V = int(log_uniform(1000, 151936))
    pad = rng.choice([64, 64, 8, 1])
    V = V // pad * pad
    pad = rng.choice([64, 64, 8])
    dim = int(log_uniform(64, 4096)) // pad * pad
    rows = int(log_uniform(1, 8192))
    return _head(op, rows, V, dim, rng.choice([1.0, 1.0, 0.7, 1.3]), rng.choice([0.0, 0.1, 0.4]), rng.random() < 0.75, rng.random() < 0.5,
                 rng.choice([0.0, 0.0, 0.1]), rng.choice([0.0, 0.0, 1e-4]))


def work(case):
    if case["op"] == "adamw":
        n = case["elements"]
        p, g, s = (2 if case["param"] == "bf16" else 4), (2 if case["grad"] == "bf16" else 4), case["bits"] // 8
        scales = 16.0 * n / BLOCK if case["bits"] == 8 else 0.0
        return {"bytes": float(n * (2 * p + g + 4 * s + (2 if case["copy"] else 0)) + scales), "flops": 16.0 * n}
    N, V, D = case["rows"], case["V"], case["dim"]
    active = N - int(N * case["masked"])
    read, written = 2.0 * (active * D + V * D) + 8 * N, 8.0 * N
    products = 1
    if case["train"]:
        written += 2.0 * (N * D + V * D)
        products = 3
    return {"bytes": read + written, "flops": 2.0 * products * active * V * D}


# ------------------------------------------------------------------------------------ preparation

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return _prepare_adamw(case, gen) if case["op"] == "adamw" else _prepare_head(case, gen)


def _prepare_head(case, gen):
    """Logits about s N(0,1) - ln(rank), s from 1 (flat) to 4 (peaked); each row's token is sampled from its distribution."""
    N, V, D, T = case["rows"], case["V"], case["dim"], case["T"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # one direction of the hidden states carries the tokens' frequencies
    u = normal(D)
    u /= u.norm()
    lnrank = torch.log(torch.randperm(V, generator=gen, device="cuda").float() + 1.0)
    w = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 26) // D)
    for a in range(0, V, step):
        b = min(V, a + step)
        w[a:b] = normal(b - a, D) / math.sqrt(D) - lnrank[a:b, None] * u
    h = normal(N, D)
    h = ((h - (h @ u)[:, None] * u) * (1.0 + 3.0 * torch.rand((N, 1), generator=gen, device="cuda")) + u).bfloat16()
    x = torch.empty(N, dtype=torch.int64, device="cuda")
    step = max(1, (1 << 27) // V)
    for a in range(0, N, step):
        b = min(N, a + step)
        y = (h[a:b] @ w.t()).float().div_(T)
        g = torch.rand((b - a, V), generator=gen, device="cuda").clamp_(min=1e-10, max=1 - 1e-7)
        x[a:b] = (y - torch.log(-torch.log(g))).argmax(-1)
    x[torch.randperm(N, generator=gen, device="cuda")[:int(N * case["masked"])]] = -100
    st = dict(case=case, h=h, w=w, x=x.int())
    active = (x >= 0).sum().clamp(min=1)
    if case["op"] == "head_logprob_grad":
        # what the forward pass gave the caller (in pieces: logits in 32 bits), and dL/dl, dL/dH of a mean over the rows
        lse, H = [], []
        for a in range(0, N, step):
            y = (h[a:a + step].float() @ w.float().t()).div_(T)
            s = torch.logsumexp(y, -1)
            lse.append(s)
            H.append(s - (torch.exp(y - s[:, None]) * y).sum(-1))
        st["lse"], st["H"] = torch.cat(lse), torch.cat(H)
        st["dl"] = normal(N) / active
        st["dH"] = torch.full((N,), -0.01, device="cuda") / active if case["entropy"] else None
    elif case["op"] == "head_cross_entropy":
        st["row_weight"] = (0.5 + torch.rand(N, generator=gen, device="cuda")) / active
    return st


def _sizes(case):
    n, total = case["tensors"], case["elements"]
    if case["sizes"] == "even":
        share = [1.0] * n
    else:                                          # two large ones (embedding, head), matrices, and as many norms and biases
        share = [(0.2 if i < 2 else 1.0 / n if i % 2 else 1e-5) for i in range(n)]
    sizes = [max(1, int(total * s / sum(share))) for s in share]
    sizes[0] = max(1, sizes[0] + total - sum(sizes))
    return sizes


def _prepare_adamw(case, gen):
    """Tensors as views of flat buffers, each from a multiple of 256 elements on, as a trainer lays them out; zeros between them."""
    n = _sizes(case)
    start = [0]
    for k in n:
        start.append(start[-1] + k + -k % BLOCK)
    total, P, G = start[-1], _TYPES[case["param"]], _TYPES[case["grad"]]

    def normal():
        return torch.randn(total, generator=gen, device="cuda")

    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, k in zip(start, n):
        inside[a:a + k] = True
    # gradients of elements over three decades of size; the states of a step that is under way
    size = torch.exp(2.0 * normal()).mul_(1e-3).mul_(inside)
    flat = dict(param=normal().mul_(0.02).mul_(inside).to(P), grad=normal().mul_(size).to(G))
    m, v = normal().mul_(size).mul_(0.3), torch.rand(total, generator=gen, device="cuda").add_(0.5).mul_(size).mul_(size).mul_(0.25)
    del size, inside
    if case["bits"] == 8:
        m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
        flat["avg_scale"], flat["sq_scale"] = m.abs().amax(-1) / M_MAX, v.amax(-1) / V_MAX
        m, v = m / flat["avg_scale"][:, None], v / flat["sq_scale"][:, None]
        m, v = m.view(-1).to(torch.float8_e4m3fn), v.view(-1).to(torch.float8_e5m2)
    flat.update(exp_avg=m, exp_avg_sq=v)
    if case["copy"]:
        flat["param_copy"] = flat["param"].bfloat16()
    tensors = []
    for a, k in zip(start, n):
        t = {key: f[a // BLOCK:(a + k + -k % BLOCK) // BLOCK] if "scale" in key else f[a:a + k] for key, f in flat.items()}
        tensors.append(dict(t, weight_decay=0.1 if k > 4096 else 0.0))
    return dict(case=case, flat=flat, tensors=tensors, start=start)


_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------ one pass

def run(st):
    if st["case"]["op"] == "adamw":
        return _run_adamw_own(st) if own else _run_adamw_plain(st)
    return _run_head_own(st) if own else _run_head_plain(st)


@functools.lru_cache(maxsize=None)
def _context(V, T):
    """The handle that a program keeps for its model's vocabulary."""
    import paper_2512_11280_b200 as adasd
    c = adasd.Context(1, V, 1, adasd.ADASD_BF16, list_capacity=1)
    c.set_warpers(T)
    return c


def _keep(st):
    """What a program that makes these calls keeps beside its inputs: handle, scratch and output buffers, or the tensors' table."""
    c = st["case"]
    if c["op"] == "adamw":
        st["ctx"] = _context(1000, 1.0)
        st["table"] = st["ctx"].adamw_table(st["tensors"])
        return
    N, ctx = c["rows"], _context(c["V"], c["T"])
    train = c["train"]
    f32 = dict(dtype=torch.float32, device="cuda")
    st["ctx"] = ctx
    st["out"] = {k: torch.empty(n, **f32) for k, n in (("logp", N), ("H", N), ("row_loss", N), ("loss", 1))}
    st["out"].update(grad_h=torch.empty_like(st["h"]) if train else None, grad_w=torch.empty_like(st["w"]) if train else None)
    st["scratch"] = torch.empty(ctx.head_scratch(N, c["dim"], grad=train), dtype=torch.uint8, device="cuda")


def _run_head_own(st):
    if "ctx" not in st:
        _keep(st)
    c, ctx, o = st["case"], st["ctx"], st["out"]
    if c["op"] == "head_logprob":
        ctx.head_logprob(st["h"], st["w"], st["x"], o["logp"], st["scratch"], entropy_out=o["H"] if c["entropy"] else None)
        return {k: o[k] for k in (("logp", "H") if c["entropy"] else ("logp",))}
    if c["op"] == "head_logprob_grad":
        ctx.head_logprob_grad(st["h"], st["w"], st["x"], st["lse"], st["dl"], st["scratch"], entropy=st["H"] if c["entropy"] else None,
                              grad_entropy=st["dH"], grad_hidden_out=o["grad_h"], grad_weight_out=o["grad_w"])
        return {k: o[k] for k in ("grad_h", "grad_w")}
    ctx.head_cross_entropy(st["h"], st["w"], st["x"], o["row_loss"], st["scratch"], row_weight=st["row_weight"], label_smoothing=c["smoothing"],
                           z_loss=c["z_loss"], loss_out=o["loss"], logp_out=o["logp"], grad_hidden_out=o["grad_h"], grad_weight_out=o["grad_w"])
    return {k: o[k] for k in ("loss", "row_loss", "logp") + (("grad_h", "grad_w") if c["train"] else ())}


def _run_head_plain(st):
    c, V = st["case"], st["w"].shape[0]
    on = (st["x"] >= 0) & (st["x"] < V)
    x = torch.where(on, st["x"], 0).long()[:, None]
    h, w = torch.where(on[:, None], st["h"].float(), 0.0), st["w"].float()
    t = (h @ w.t()) / c["T"]
    m = t.amax(-1, keepdim=True)
    t -= m                                          # z less the row's largest
    e = torch.exp(t)
    S = e.sum(-1, keepdim=True)
    lnS = torch.log(S)
    l, lse = (t.gather(1, x) - lnS)[:, 0], (m + lnS)[:, 0]
    p = e.div_(S)
    off = lambda v: torch.where(on, v, 0.0)  # noqa: E731
    if c["op"] == "head_logprob":
        got = {"logp": off(l)}
        if c["entropy"]:
            got["H"] = off(lnS[:, 0] - (p * t).sum(-1))
        return got
    got = {}
    if c["op"] == "head_logprob_grad":
        a, b, const = -off(st["dl"]), off(st["dl"]), 0.0
        if c["entropy"]:
            dH = off(st["dH"])
            g = p * (a[:, None] - dH[:, None] * ((t - lnS) + st["H"][:, None]))
        else:
            g = p * a[:, None]
    else:
        rw, s = off(st["row_weight"]), c["smoothing"]
        loss = -(1.0 - s) * l
        if s:
            loss = loss - s * (t.mean(-1) - lnS[:, 0])
        if c["z_loss"]:
            loss = loss + c["z_loss"] * lse * lse
        loss = off(loss * rw)
        got.update(loss=loss.sum()[None], row_loss=loss, logp=off(l))
        if not c["train"]:
            return got
        b, const = -(1.0 - s) * rw, -s / V * rw
        g = p * (rw * (1.0 + 2.0 * c["z_loss"] * lse))[:, None] + const[:, None]
    del t, p, e
    g.scatter_add_(1, x, b[:, None])
    g /= c["T"]
    got["grad_h"], got["grad_w"] = (g @ w).bfloat16(), (g.t() @ h).bfloat16()
    return got


def _run_adamw_own(st):
    if "ctx" not in st:
        _keep(st)
    st["ctx"].adamw_step(st["table"], lr=LR, step=STEP, betas=(BETA1, BETA2), eps=EPS, grad_scale=GRAD_SCALE,
                         rounding="stochastic" if st["case"]["stochastic"] else "nearest", seed=SEED)
    return _adamw_outputs(st)


def _adamw_outputs(st):
    return {k: f for k, f in st["flat"].items() if k != "grad"}


def _mix(x):
    """A mixing function of 32-bit integers (held in 64)."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _noise(i, n):
    key = _mix(SEED ^ _mix((STEP + 0x9E3779B9 * (i + 1)) & 0xFFFFFFFF))
    return _mix((torch.arange(n, device="cuda") + key) & 0xFFFFFFFF)


def _to_grid(y, bits, dropped, least):
    """|y| moved down to a value of a small float, after its dropped bits (of `least`'s steps below the smallest normal) had
    `bits` / 2^20 (2^21) of a step added to them."""
    a = y.abs()
    big = ((a.view(torch.int32) + bits.int()) & -(1 << dropped)).view(torch.float32)
    small = torch.floor(a / least + bits.float() * (0.5 ** dropped)) * least
    return torch.where(a < least * 2 ** (23 - dropped), small, big).copysign(y)


def _run_adamw_plain(st):
    c, f, start = st["case"], st["flat"], st["start"]
    eight = c["bits"] == 8
    n = [b - a for a, b in zip(start, start[1:])]
    p, g, m, v = f["param"].float(), f["grad"].float() * GRAD_SCALE, f["exp_avg"].float(), f["exp_avg_sq"].float()
    if eight:
        m = (m.view(-1, BLOCK) * f["avg_scale"][:, None]).view(-1)
        v = (v.view(-1, BLOCK) * f["sq_scale"][:, None]).view(-1)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    keep = torch.repeat_interleave(torch.tensor([1.0 - LR * t["weight_decay"] for t in st["tensors"]], device="cuda"), torch.tensor(n, device="cuda"))
    denom = torch.sqrt(v) * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + EPS
    p = p * keep - (LR / (1.0 - BETA1 ** STEP)) * (m / denom)
    noise = torch.cat([_noise(i, k) for i, k in enumerate(n)]) if c["stochastic"] and (eight or c["param"] == "bf16") else None
    if noise is not None and c["param"] == "bf16":
        hi = ((noise * 0x9E3779B1) & 0xFFFFFFFF) >> 16
        p = ((p.view(torch.int32) + hi.int()) & -65536).view(torch.float32)
    if eight:
        m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
        m_top, v_top = m.abs().amax(-1, keepdim=True), v.amax(-1, keepdim=True)
        f["avg_scale"].copy_((m_top * (1.0 / M_MAX))[:, 0])
        f["sq_scale"].copy_((v_top * (1.0 / V_MAX))[:, 0])
        # (number / tensor would be a reciprocal and a product; a block of nothing but tiny values is held as zeros)
        y = m * torch.where(m_top >= LEAST, torch.full_like(m_top, M_MAX) / m_top, 0.0)
        q = v * torch.where(v_top >= LEAST, torch.full_like(v_top, V_MAX) / v_top, 0.0)
        if noise is not None:
            y = _to_grid(y, (noise & 0xFFFFF).view(-1, BLOCK), 20, 2.0 ** -9)
            q = _to_grid(q, (noise >> 11).view(-1, BLOCK), 21, 2.0 ** -16)
        m = y.clamp(-M_MAX, M_MAX).to(torch.float8_e4m3fn).view(-1)
        q = q.clamp(max=V_MAX).to(torch.float8_e5m2).view(torch.uint8)
        v = torch.where((v > 0) & (q == 0), 1, q.int()).to(torch.uint8).view(torch.float8_e5m2).view(-1)
    f["param"].copy_(p)
    f["exp_avg"].copy_(m)
    f["exp_avg_sq"].copy_(v)
    if c["copy"]:
        f["param_copy"].copy_(p)
    return _adamw_outputs(st)


# ------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """The same from the definitions in 64 bits, every gradient by differentiating the loss."""
    st = prepare(case, seed)
    return _exact_adamw(st) if case["op"] == "adamw" else _exact_head(st)


def _exact_head(st):
    c, N, V, D = st["case"], st["case"]["rows"], st["case"]["V"], st["case"]["dim"]
    train = c["train"]
    w = st["w"].double()
    on = st["x"] >= 0
    x = st["x"].long().clamp(min=0)
    step = max(1, (1 << 28) // V)
    parts = {}
    grad_w = torch.zeros((V, D), dtype=torch.float64, device="cuda") if train else None
    for a in range(0, N, step):
        b = min(N, a + step)
        h = st["h"][a:b].double()
        z = (h @ w.t()).requires_grad_(train)
        v = z / c["T"]
        lse = torch.logsumexp(v, -1)
        l = torch.where(on[a:b], v.gather(1, x[a:b, None])[:, 0] - lse, 0.0)
        new, total = {}, None
        if c["entropy"] and c["op"] != "head_cross_entropy":
            H = torch.where(on[a:b], lse - (torch.softmax(v, -1) * v).sum(-1), 0.0)
        if c["op"] == "head_logprob":
            new["logp"] = l
            if c["entropy"]:
                new["H"] = H
        elif c["op"] == "head_logprob_grad":
            total = (l * st["dl"][a:b].double()).sum()
            if c["entropy"]:
                total = total + (H * st["dH"][a:b].double()).sum()
        else:
            s = c["smoothing"]
            loss = -(1 - s) * l + c["z_loss"] * lse ** 2
            if s:
                loss = loss - s * (v.mean(-1) - lse)
            new["row_loss"] = torch.where(on[a:b], loss * st["row_weight"][a:b].double(), 0.0)
            new["logp"] = l
            total = new["row_loss"].sum()
        if train:
            g = torch.autograd.grad(total, z)[0]
            new["grad_h"] = g @ w
            grad_w.addmm_(g.t(), h)
            del g
        del z, v
        for k, t in new.items():
            parts.setdefault(k, []).append(t.detach())
    got = {k: torch.cat(v) for k, v in parts.items()}
    if c["op"] == "head_cross_entropy":
        got = {"loss": got["row_loss"].sum()[None], **got}
    if train:
        got["grad_w"] = grad_w
    return got


def _exact_adamw(st):
    c, f = st["case"], st["flat"]
    m, v, g = f["exp_avg"].double(), f["exp_avg_sq"].double(), f["grad"].double() * GRAD_SCALE
    if c["bits"] == 8:
        m = m * f["avg_scale"].double().repeat_interleave(BLOCK)
        v = v * f["sq_scale"].double().repeat_interleave(BLOCK)
    m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g ** 2 - v)
    del g
    p = f["param"].double()
    for t, a in zip(st["tensors"], st["start"]):
        p[a:a + t["param"].numel()] *= 1 - LR * t["weight_decay"]
    p -= LR * (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    got = {k: None for k in _adamw_outputs(st)}
    got["param"] = p
    if c["copy"]:
        got["param_copy"] = p
    if c["bits"] == 8:                              # the states' values are what rounding makes of them; the scales are not rounded
        got["avg_scale"] = m.view(-1, BLOCK).abs().amax(-1) / M_MAX
        got["sq_scale"] = v.view(-1, BLOCK).amax(-1) / V_MAX
    else:
        got.update(exp_avg=m, exp_avg_sq=v)
    return got
