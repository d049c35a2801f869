"""Scoring and training on given tokens: the cases that these operators are measured on, their plain form in
elementary torch operations, and their values in 64 bits.

A row is a position's logits z over the vocabulary, x the token that stands there, T the temperature that the
sequences were sampled at.  l = ln softmax(z / T)_x, H the row's entropy.  A row whose token is negative is left out
(a prompt, padding): it is not read, counts nothing and has a gradient of zeros.

  token_logprob     l and H of every row; train: the gradient of a loss with given dL/dl and dL/dH
  policy_loss       clipped policy loss: ratio exp(l - l_old), advantage, clip range, KL estimate e^r - r - 1 with
                    r = l_ref - l, entropy bonus; the weighted sum over the rows and its gradient
  preference_loss   pairs of packed sequences, chosen and rejected: the log ratios' difference
                    D = (l_c - ref_c) - (l_r - ref_r), -ln sigma(beta D) or (D - 1/(2 beta))^2, and its gradient

A case:
  op       "token_logprob", "policy_loss" or "preference_loss"
  rows, V  rows of logits (of all sequences together) and vocabulary
  dtype    "bf16" or "fp32" logits and gradients
  T        temperature
  masked   share of the rows that are left out
  train    with the gradient; else the forward pass alone
  entropy  token_logprob: H too; policy_loss: an entropy bonus
  kl       policy_loss: with the KL term
  pairs, squared, average   preference_loss: pairs, the squared loss, log-probs averaged over a sequence's rows
"""
import functools
import math

import torch

own = False

CLIP_LOW, CLIP_HIGH, KL_COEF, ENT_COEF = 0.2, 0.28, 0.04, 0.01
BETA, SMOOTHING = 0.1, 0.05


def _case(op, rows, V, dtype="bf16", T=1.0, masked=0.0, train=True, entropy=False, kl=False, pairs=0, squared=False,
          average=False, name=None):
    c = dict(op=op, rows=rows, V=V, dtype=dtype, T=T, masked=masked, train=train, entropy=entropy, kl=kl, pairs=pairs,
             squared=squared, average=average)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of one request whose caller asked for log-probs: latency
        _case("token_logprob", 1, 32000, train=False, entropy=True, name="logprob one token"),
        # one verification round of an ordinary batch (B=32, K=8), its tokens scored
        _case("token_logprob", 288, 128256, train=False, entropy=True, name="logprob round"),
        # sequences scored by a reference model ahead of training
        _case("token_logprob", 4096, 151936, masked=0.25, train=False, name="logprob sequences"),
        # a loss of the user's own on log-probs and entropies, vocabulary of no round size, rows packed
        _case("token_logprob", 1000, 50257, entropy=True, name="logprob gradient odd"),
        # one short sequence of a small model with fp32 logits
        _case("policy_loss", 7, 32000, "fp32", kl=True, name="policy short fp32"),
        # a micro-batch of ordinary length, sampled at temperature 0.8
        _case("policy_loss", 2048, 128256, T=0.8, masked=0.1, kl=True, name="policy micro-batch"),
        # the largest: long packed sequences, a quarter of the rows prompts, every term
        _case("policy_loss", 4096, 151936, masked=0.25, entropy=True, kl=True, name="policy packed"),
        # fp32 logits of a large vocabulary
        _case("policy_loss", 517, 128256, "fp32", name="policy fp32"),
        # the loss alone, as an evaluation reports it
        _case("policy_loss", 999, 128256, train=False, entropy=True, kl=True, name="policy evaluation"),
        # one pair of short answers of a small model
        _case("preference_loss", 61, 32000, pairs=1, name="preference one pair"),
        # a micro-batch of pairs of ragged lengths, a quarter of the rows prompts
        _case("preference_loss", 3300, 128256, masked=0.25, pairs=8, name="preference micro-batch"),
        # fp32, squared loss on averaged log-probs, vocabulary of no round size
        _case("preference_loss", 801, 50257, "fp32", pairs=5, squared=True, average=True, name="preference fp32 odd"),
    ]


def draw(rng):
    def log_uniform(a, b):
        return math.exp(rng.uniform(math.log(a), math.log(b)))
    op = rng.choice(["token_logprob", "policy_loss", "policy_loss", "preference_loss"])
    V = int(log_uniform(1000, 151936))
    pad = rng.choice([64, 64, 8, 1])
    V = V // pad * pad
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    pairs = int(log_uniform(1, 16)) if op == "preference_loss" else 0
    rows = max(int(log_uniform(1, 8192)), 2 * pairs)
    most = 2.4e9 / (2 * V * (2 if dtype == "bf16" else 4))
    rows = max(1, 2 * pairs, min(rows, int(most)))
    return _case(op, rows, V, dtype, rng.choice([1.0, 1.0, 0.7, 1.3]), rng.choice([0.0, 0.1, 0.4]), rng.random() < 0.75,
                 rng.random() < 0.5, rng.random() < 0.5, pairs, rng.random() < 0.3, rng.random() < 0.3)


def work(case):
    N, V, e = case["rows"], case["V"], 2 if case["dtype"] == "bf16" else 4
    active = N - int(N * case["masked"])
    read, written = active * V * e + 24 * N, 12 * N
    flops = 4.0 * active * V
    if case["train"]:
        written += N * V * e
        flops *= 2
    return {"bytes": float(read + written), "flops": flops}


# ------------------------------------------------------------------------------------ preparation

@functools.lru_cache(maxsize=None)
def _context(V, dtype, T):
    """The handle that a program keeps for its model's vocabulary."""
    import paper_2512_11280_b200 as adasd
    c = adasd.Context(1, V, 1, adasd.ADASD_BF16 if dtype == "bf16" else adasd.ADASD_FP32, list_capacity=1)
    c.set_warpers(T)
    return c


def _rows(case, gen):
    """Rows s N(0,1) - ln(rank), s from 1 (flat) to 6 (peaked), and a token of each, sampled from it."""
    N, V, T = case["rows"], case["V"], case["T"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    lnrank = torch.log(torch.randperm(V, generator=gen, device="cuda").float() + 1.0)
    z, x = torch.empty((N, V), dtype=dt, device="cuda"), torch.empty(N, dtype=torch.int64, device="cuda")
    l = torch.empty(N, dtype=torch.float64, device="cuda")
    s = 1.0 + 5.0 * torch.rand((N, 1), generator=gen, device="cuda")   # flat to peaked
    step = max(1, (1 << 26) // V)
    for a in range(0, N, step):
        b = min(N, a + step)
        y = torch.randn((b - a, V), generator=gen, device="cuda").mul_(s[a:b]).sub_(lnrank)
        z[a:b] = y
        y = z[a:b].float().div_(T)
        l[a:b] = -torch.logsumexp(y, -1).double()
        g = torch.rand((b - a, V), generator=gen, device="cuda").clamp_(min=1e-10, max=1 - 1e-7)
        x[a:b] = (y - torch.log(-torch.log(g))).argmax(-1)
        l[a:b] += y.gather(1, x[a:b, None])[:, 0].double()
    return z, x, l


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    N, P = case["rows"], case["pairs"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    z, x, l = _rows(case, gen)
    x[torch.randperm(N, generator=gen, device="cuda")[:int(N * case["masked"])]] = -100
    st = dict(case=case, z=z, x=x.int(), grad=torch.empty_like(z) if case["train"] else None)
    f32 = dict(dtype=torch.float32, device="cuda")
    active = (x >= 0).sum().clamp(min=1)
    if case["op"] == "token_logprob":
        if case["train"]:                      # dL/dl and dL/dH as a mean over the rows gives them
            st["a"] = (normal(N) / active).float()
            st["b"] = (-0.01 / active * torch.ones(N, **f32)) if case["entropy"] else None
    elif case["op"] == "policy_loss":
        # advantages over a baseline that lags behind; behaviour and reference log-probs are near the policy's
        st["adv"] = 0.3 + normal(N)
        d = 0.2 * normal(N).double()
        ratio = torch.exp(-d)
        for edge in (1 - CLIP_LOW, 1 + CLIP_HIGH):       # (a ratio at the very edge of the clip range may go either way)
            d = torch.where((ratio - edge).abs() < 1e-4, d + 1e-3, d)
        st["old"] = (l + d).float()
        st["ref"] = (l + 0.3 * normal(N).double()).float() if case["kl"] else None
        st["w"] = torch.ones(N, **f32) / active
    else:
        # 2 P packed sequences of ragged lengths, the P chosen ones first
        share = torch.rand(2 * P, generator=gen, device="cuda").double() + 0.2
        cut = (share.cumsum(0) / share.sum() * N).round().long()
        start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cut])
        start[-1] = N
        seq = torch.bucketize(torch.arange(N, device="cuda"), start[1:], right=True)
        score = _by_sequence(l * (x >= 0), (x >= 0), seq, 2 * P, case["average"])
        st["start"], st["P"] = start.int(), P
        st["ref"] = (score + (0.5 if case["average"] else 5.0) * normal(2 * P).double()).float()
    if own:
        st["ctx"] = _context(case["V"], case["dtype"], case["T"])
        st["out"] = {k: torch.empty(n, **f32) for k, n in
                     (("logp", N), ("H", N), ("kl", N), ("row_loss", N), ("loss", 1), ("seq", 2 * P), ("pair_loss", P))}
        st["scratch"] = torch.empty(16 * N + 16 * P, dtype=torch.uint8, device="cuda")
    return st


def _by_sequence(v, counted, seq, n, average):
    total = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, seq, v.double())
    if average:
        total = total / torch.zeros_like(total).index_add_(0, seq, counted.double()).clamp(min=1)
    return total


# ------------------------------------------------------------------------------------ one pass

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    c, ctx, o = st["case"], st["ctx"], st["out"]
    if c["op"] == "token_logprob":
        if c["train"]:
            ctx.token_logprob_grad(st["z"], st["x"], st["a"], st["grad"], grad_entropy=st["b"])
            return {"grad": st["grad"]}
        ctx.token_logprob(st["z"], st["x"], o["logp"], entropy_out=o["H"] if c["entropy"] else None)
        return {k: o[k] for k in (("logp", "H") if c["entropy"] else ("logp",))}
    if c["op"] == "policy_loss":
        ctx.policy_loss(st["z"], st["x"], st["adv"], o["row_loss"], old_logp=st["old"], ref_logp=st["ref"], weight=st["w"],
                        clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL_COEF if c["kl"] else 0.0,
                        entropy_coef=ENT_COEF if c["entropy"] else 0.0, loss_out=o["loss"], logp_out=o["logp"],
                        entropy_out=o["H"] if c["entropy"] else None, kl_out=o["kl"] if c["kl"] else None, grad_out=st["grad"])
        keys = ["loss", "row_loss", "logp"] + ["H"] * c["entropy"] + ["kl"] * c["kl"]
    else:
        ctx.preference_loss(st["z"], st["x"], st["start"], o["pair_loss"], o["seq"], st["scratch"], ref_logp=st["ref"],
                            rule="squared" if c["squared"] else "sigmoid", beta=BETA, average=c["average"],
                            label_smoothing=0.0 if c["squared"] else SMOOTHING, scale=1.0 / c["pairs"], loss_out=o["loss"],
                            grad_out=st["grad"])
        keys = ["loss", "pair_loss", "seq"]
    got = {k: o[k] for k in keys}
    if c["train"]:
        got["grad"] = st["grad"]
    return got


def _plain_logp(st):
    """Of every row: ln p and p in 32 bits, l in 64 (rows left out: token 0 stands in), which rows count, their tokens."""
    z = st["z"].float()
    on = (st["x"] >= 0) & (st["x"] < z.shape[1])
    x = torch.where(on, st["x"], 0).long()[:, None]
    t = (z - z.amax(-1, keepdim=True)) / st["case"]["T"]
    e = torch.exp(t)
    S = e.sum(-1, keepdim=True)
    logp = t.gather(1, x).double() - torch.log(S.double())
    return t - torch.log(S), e / S, logp[:, 0], on, x


def _plain_grad(st, lnp, p, on, x, dl, dH, H):
    """dL/dz from dL/dl and dL/dH of every row."""
    g = -dl.float()[:, None] * p
    g.scatter_add_(1, x, dl.float()[:, None])
    if dH is not None:
        g -= dH.float()[:, None] * p * (lnp + H.float()[:, None])
    return torch.where(on[:, None], g / st["case"]["T"], 0.0).to(st["z"].dtype)


def _run_plain(st):
    c = st["case"]
    lnp, p, l, on, x = _plain_logp(st)
    H = -(p * lnp).sum(-1) if c["entropy"] and c["op"] != "preference_loss" else None
    got = {}
    if c["op"] == "token_logprob":
        if c["train"]:
            return {"grad": _plain_grad(st, lnp, p, on, x, st["a"], st["b"], H)}
        got["logp"] = torch.where(on, l, 0.0).float()
        if c["entropy"]:
            got["H"] = torch.where(on, H, 0.0).float()
        return got
    if c["op"] == "policy_loss":
        A, w = st["adv"].double(), torch.where(on, st["w"], 0.0).double()
        ratio = torch.exp(l - st["old"].double())
        s1, s2 = ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A
        loss, dl = -torch.minimum(s1, s2), torch.where(s1 <= s2, -s1, 0.0)
        if c["kl"]:
            r = st["ref"].double() - l
            k3 = torch.exp(r) - r - 1
            loss, dl = loss + KL_COEF * k3, dl + KL_COEF * (1 - torch.exp(r))
            got["kl"] = torch.where(on, k3, 0.0).float()
        if c["entropy"]:
            loss = loss - ENT_COEF * H
            got["H"] = torch.where(on, H, 0.0).float()
        loss = torch.where(on, loss * w, 0.0)
        got.update(loss=loss.sum()[None].float(), row_loss=loss.float(), logp=torch.where(on, l, 0.0).float())
        if c["train"]:
            got["grad"] = _plain_grad(st, lnp, p, on, x, dl * w, -ENT_COEF * w if c["entropy"] else None, H)
        return got
    P, start = st["P"], st["start"].long()
    seq = torch.bucketize(torch.arange(l.numel(), device="cuda"), start[1:], right=True)
    total = _by_sequence(torch.where(on, l, 0.0), on, seq, 2 * P, c["average"])
    d = total - st["ref"].double()
    D = d[:P] - d[P:]
    if c["squared"]:
        loss, dD = (D - 0.5 / BETA) ** 2, 2 * (D - 0.5 / BETA)
    else:
        u = BETA * D
        s = 1 / (1 + torch.exp(-u))
        loss = (1 - SMOOTHING) * torch.log1p(torch.exp(-u)) + SMOOTHING * torch.log1p(torch.exp(u))
        dD = BETA * (s - (1 - SMOOTHING))
    got.update(loss=(loss / P).sum()[None].float(), pair_loss=(loss / P).float(), seq=total.float())
    if c["train"]:
        per = torch.cat([dD, -dD]) / P
        if c["average"]:
            per = per / torch.zeros_like(per).index_add_(0, seq, on.double()).clamp(min=1)
        got["grad"] = _plain_grad(st, lnp, p, on, x, torch.where(on, per[seq], 0.0), None, None)
    return got


# ------------------------------------------------------------------------------------ in 64 bits

def _chunks(N, V):
    step = max(1, (1 << 25) // V)
    return [(a, min(N, a + step)) for a in range(0, N, step)]


def exact(case, seed):
    """The same from the definitions in 64 bits: log-probs from logsumexp, every gradient by differentiating the loss."""
    st = prepare(case, seed)
    c, z, N, V = case, st["z"], case["rows"], case["V"]
    on = st["x"] >= 0
    x = st["x"].long().clamp(min=0)
    grad = torch.zeros((N, V), dtype=torch.float64, device="cuda") if c["train"] else None

    def scores(a, b, entropy):
        y = z[a:b].double().requires_grad_(c["train"])
        v = y / c["T"]
        lse = torch.logsumexp(v, -1)
        l = torch.where(on[a:b], v.gather(1, x[a:b, None])[:, 0] - lse, 0.0)
        H = torch.where(on[a:b], lse - (torch.softmax(v, -1) * v).sum(-1), 0.0) if entropy else None
        return y, l, H

    def differentiate(total, y, a, b):
        grad[a:b] = torch.autograd.grad(total, y)[0]

    if c["op"] == "preference_loss":
        P, start = st["P"], st["start"].tolist()
        l = torch.cat([scores(a, b, False)[1].detach() for a, b in _chunks(N, V)]).requires_grad_(c["train"])
        total = []
        for s in range(2 * P):
            a, b = start[s], start[s + 1]
            total.append(l[a:b].sum() / max(1, int(on[a:b].sum())) if c["average"] else l[a:b].sum())
        total = torch.stack(total)
        d = total - st["ref"].double()
        D = d[:P] - d[P:]
        if c["squared"]:
            loss = (D - 1 / (2 * BETA)) ** 2
        else:
            ls = torch.nn.functional.logsigmoid
            loss = -(1 - SMOOTHING) * ls(BETA * D) - SMOOTHING * ls(-BETA * D)
        loss = loss / P
        got = dict(loss=loss.sum()[None].detach(), pair_loss=loss.detach(), seq=total.detach())
        if c["train"]:
            dl = torch.autograd.grad(loss.sum(), l)[0]
            for a, b in _chunks(N, V):
                y, lc, _ = scores(a, b, False)
                differentiate((lc * dl[a:b]).sum(), y, a, b)
            got["grad"] = grad
        return got

    parts = {}
    for a, b in _chunks(N, V):
        y, l, H = scores(a, b, c["entropy"])
        if c["op"] == "token_logprob":
            if c["train"]:
                total = (st["a"][a:b].double() * l).sum()
                if c["entropy"]:
                    total = total + (st["b"][a:b].double() * H).sum()
                differentiate(total, y, a, b)
                continue
            new = dict(logp=l, H=H)
        else:
            A = st["adv"][a:b].double()
            ratio = torch.exp(l - st["old"][a:b].double())
            loss = -torch.minimum(ratio * A, torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * A)
            new = dict(logp=l, H=H, kl=None)
            if c["kl"]:
                r = st["ref"][a:b].double() - l
                new["kl"] = torch.where(on[a:b], torch.expm1(r) - r, 0.0)
                loss = loss + KL_COEF * new["kl"]
            if c["entropy"]:
                loss = loss - ENT_COEF * H
            new["row_loss"] = torch.where(on[a:b], loss * st["w"][a:b].double(), 0.0)
            if c["train"]:
                differentiate(new["row_loss"].sum(), y, a, b)
        for k, v in new.items():
            if v is not None:
                parts.setdefault(k, []).append(v.detach())
    got = {k: torch.cat(v) for k, v in parts.items()}
    if c["op"] == "policy_loss":
        got["loss"] = got["row_loss"].sum()[None]
    if c["train"]:
        got["grad"] = grad
    return got
