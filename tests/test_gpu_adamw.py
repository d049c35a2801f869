"""The AdamW step against 64 bits; its 8-bit states against the same formats in elementary operations, code by code."""
import pytest

from tests import adamw_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return torch


@pytest.fixture(scope="module")
def ctx(torch):
    import paper_2512_11280_b200 as adasd
    return adasd.Context(1, 100, 1, list_capacity=1)


def cut(torch, values, offset):
    """The values as a view that starts `offset` elements into an allocation of sevens."""
    n = values.numel()
    buf = torch.full((n + offset + 64,), 7.0, device="cuda").to(values.dtype)
    view = buf[offset:offset + n]
    view.copy_(values)
    return view, buf


def tensor(torch, n, g, param="float32", grad="float32", bits=32, copy=False, wd=0.1, offset=0, fresh=False):
    """A tensor in mid-training and the buffers that its arrays are views of."""
    rnd = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    size = 1e-3 * torch.exp(2 * rnd())
    m, v = 0.3 * size * rnd(), size * size * 0.25
    if fresh:
        m, v = 0 * m, 0 * v
    a = dict(param=(0.05 * rnd()).to(getattr(torch, param)), grad=(size * rnd()).to(getattr(torch, grad)))
    if bits == 8:
        pad = lambda x: torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)  # noqa: E731
        a["avg_scale"], a["sq_scale"] = pad(m).abs().amax(-1) / 448, pad(v).amax(-1) / 57344
        full = lambda s: s.repeat_interleave(256)[:n].clamp(min=1e-30)  # noqa: E731
        a["exp_avg"], a["exp_avg_sq"] = (m / full(a["avg_scale"])).to(torch.float8_e4m3fn), (v / full(a["sq_scale"])).to(torch.float8_e5m2)
    else:
        a["exp_avg"], a["exp_avg_sq"] = m, v
    if copy:
        a["param_copy"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    views, bufs = {}, {}
    for k, x in a.items():
        views[k], bufs[k] = cut(torch, x, offset)
    views["weight_decay"] = wd
    return views, bufs


def same(torch, x, y):
    return torch.equal(x.view(torch.uint8) if x.dtype.itemsize == 1 else x, y.view(torch.uint8) if y.dtype.itemsize == 1 else y)


def before(t):
    return {k: (v.clone() if hasattr(v, "clone") else v) for k, v in t.items()}


OPT = dict(lr=1e-2, step=7, betas=(0.9, 0.999), eps=1e-8, grad_scale=0.375)


def check(torch, old, t, index=0, rounding="nearest", seed=0, lr=1e-2, step=7, betas=(0.9, 0.999), eps=1e-8, grad_scale=0.375):
    n = t["param"].numel()
    p, m, v, tp, tm, tv = ref.step(old, lr, step, *betas, eps, grad_scale)
    half = 0.0 if t["param"].dtype is torch.float32 else 2.0 ** -8 if rounding == "nearest" else 2.0 ** -7
    d = (t["param"].double() - p).abs()
    assert bool((d <= tp + half * (p.abs() + tp)).all()), float((d / (tp + half * p.abs())).max())
    if "param_copy" in t:
        assert torch.equal(t["param_copy"], t["param"].bfloat16())
    if t["exp_avg"].dtype is torch.float32:
        assert bool(((t["exp_avg"].double() - m).abs() <= tm).all()) and bool(((t["exp_avg_sq"].double() - v).abs() <= tv).all())
    else:
        h = ref.noise(n, seed, step, index, "cuda") if rounding == "stochastic" else None
        want = ref.codes(old, *betas, grad_scale, h)
        for k, w in zip(("exp_avg", "exp_avg_sq", "avg_scale", "sq_scale"), want):
            got = t[k].view(torch.uint8) if t[k].dtype.itemsize == 1 else t[k]
            assert torch.equal(got, w), (k, int((got != w).sum()))
    assert same(torch, t["grad"], old["grad"])


@pytest.mark.parametrize("param,grad", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
def test_every_type_and_length(torch, ctx, param, grad, bits, rounding):
    """Lengths about a lane's elements, a block, an item; at 16-byte boundaries and off them; what lies around the arrays stays."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for n in (1, 7, 8, 31, 255, 256, 257, 2047, 2048, 2049, 100003):
        for offset in (0, 1, 5):
            t, bufs = tensor(torch, n, g, param, grad, bits, copy=param == "float32", offset=offset)
            old = before(t)
            ctx.adamw_step(ctx.adamw_table([t]), rounding=rounding, seed=5, **OPT)
            check(torch, old, t, 0, rounding, 5)
            for k, b in bufs.items():
                rest = torch.cat([b[:offset], b[offset + t[k].numel():]]).float()
                assert bool((rest == rest[0]).all()) and abs(float(rest[0]) - 7) < 0.1, k
    assert ctx.status() == 0


@pytest.mark.parametrize("count", [2, 24, 25, 384, 385, 800])
def test_many_tensors_of_all_kinds(torch, ctx, count):
    """More than a launch takes; every tensor has its own weight decay and its own place in the hash."""
    g = torch.Generator(device="cuda").manual_seed(count)
    tensors = []
    for i in range(count):
        n = (1, 300, 0, 2500, 64, 9000)[i % 6]
        tensors.append(tensor(torch, n, g, ("float32", "bfloat16")[i % 2], ("bfloat16", "float32")[i // 2 % 2], (32, 8)[i // 4 % 2],
                              copy=i % 4 == 0, wd=0.01 * (i % 5), offset=(0, 0, 3)[i % 3])[0])
    old = [before(t) for t in tensors]
    ctx.adamw_step(ctx.adamw_table(tensors), rounding="stochastic", seed=9, **OPT)
    for i, (o, t) in enumerate(zip(old, tensors)):
        if t["param"].numel():
            check(torch, o, t, i, "stochastic", 9)
    ctx.adamw_step(ctx.adamw_table([]), **OPT)
    assert ctx.status() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_first_steps_from_zero_states(torch, ctx, bits):
    g = torch.Generator(device="cuda").manual_seed(2)
    t, _ = tensor(torch, 5000, g, bits=bits, fresh=True)
    t["grad"][:600] = 0.0                        # whole blocks that no gradient reaches
    table = ctx.adamw_table([t])
    for k in (1, 2, 3):
        old = before(t)
        ctx.adamw_step(table, **dict(OPT, step=k))
        check(torch, old, t, **dict(OPT, step=k))
    assert bool((t["exp_avg"][:512].float() == 0).all()) and bool((t["exp_avg_sq"][:512].float() == 0).all())


@pytest.mark.parametrize("options", [dict(betas=(0.0, 0.0)), dict(betas=(0.95, 0.9999), step=100000), dict(eps=1e-3), dict(lr=0.0),
                                     dict(grad_scale=-1.0), dict(grad_scale=0.0)])
@pytest.mark.parametrize("bits", [32, 8])
def test_options(torch, ctx, bits, options):
    g = torch.Generator(device="cuda").manual_seed(3)
    t, _ = tensor(torch, 3000, g, bits=bits)
    old, o = before(t), {**OPT, **options}
    ctx.adamw_step(ctx.adamw_table([t]), **o)
    check(torch, old, t, **o)


def test_sizes_beyond_fp8_and_fp32(torch, ctx):
    """Blocks of tiny and of huge gradients, of one large value among zeros; no parameter that has a finite gradient moves by more than a few lr."""
    g = torch.Generator(device="cuda").manual_seed(4)
    t, _ = tensor(torch, 256 * 6, g, bits=8, fresh=True)
    t["grad"].view(6, 256)[:] = torch.tensor([1e-30, 1e-18, 1e-3, 1e3, 1e15, 0.0], device="cuda")[:, None]
    t["grad"][256 * 5 + 17] = 3.0
    t["grad"][256 * 2 + 3] = 1e8
    p0 = t["param"].clone()
    table = ctx.adamw_table([t])
    for k in range(1, 5):
        old = before(t)
        ctx.adamw_step(table, **dict(OPT, step=k))
        check(torch, old, t, **dict(OPT, step=k))
    assert float((t["param"] - p0).abs().max()) < 4 * 1.1e-2 + 4 * 1e-3
    assert ctx.status() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_what_is_not_finite_stays_where_it_is(torch, ctx, bits):
    g = torch.Generator(device="cuda").manual_seed(5)
    t, _ = tensor(torch, 1024, g, bits=bits)
    t["grad"][300], t["grad"][700] = float("nan"), float("inf")
    ctx.adamw_step(ctx.adamw_table([t]), **OPT)
    bad = ~torch.isfinite(t["param"])
    assert bool(bad[300]) and bool(bad[700]) and int(bad.sum()) == 2
    m = t["exp_avg"].float() * (t["avg_scale"].repeat_interleave(256) if bits == 8 else 1.0)
    lost = ~torch.isfinite(m).view(4, 256)
    assert not bool(lost[0].any()) and not bool(lost[3].any()) and bool(lost[1].any()) and bool(lost[2].any())


def test_rounding_up_or_down_is_right_in_the_mean(torch, ctx):
    """65536 elements of one value in every block: the mean of what is held is the value, to five standard errors (a step's size / 2 / 256)."""
    n = 1 << 16
    g = torch.Generator(device="cuda").manual_seed(6)
    t, _ = tensor(torch, n, g, "bfloat16", "float32", 8, fresh=True, wd=0.0)
    t["param"].fill_(1.0)
    t["grad"].fill_(0.013)
    t["grad"][::256] = 1.0                       # the largest of each block
    ctx.adamw_step(ctx.adamw_table([t]), **{**OPT, "lr": 1e-3, "grad_scale": 1.0, "step": 1}, rounding="stochastic", seed=3)
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[::256] = False
    m = (t["exp_avg"].double() * t["avg_scale"].double().repeat_interleave(256))[rest]
    v = (t["exp_avg_sq"].double() * t["sq_scale"].double().repeat_interleave(256))[rest]
    for got, want, step in ((m, 0.1 * 0.013, 2.0 ** -3), (v, 1e-3 * 0.013 ** 2, 2.0 ** -2), (t["param"].double()[rest], 1 - 1e-3, 2.0 ** -7)):
        assert abs(float(got.mean()) - want) < 5 * want * step / 2 / 256, (float(got.mean()), want)
    assert len(torch.unique(t["param"])) == 2


def test_values_read_on_the_device_and_replayed(torch, ctx):
    """A captured step whose rate, number and clipping factor are device scalars; the same states as steps issued one by one."""
    g = torch.Generator(device="cuda").manual_seed(7)
    a, _ = tensor(torch, 3000, g, "bfloat16", "bfloat16", 8)
    b = before(a)
    lr, step, scale = torch.tensor([1e-2], device="cuda"), torch.tensor([4], dtype=torch.int32, device="cuda"), torch.tensor([0.5], device="cuda")
    table = ctx.adamw_table([a])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.adamw_step(table, lr, step, grad_scale=0.75, grad_scale_dev=scale, rounding="stochastic", seed=11)
        step.add_(1)
    other = ctx.adamw_table([b])
    for k in range(4, 7):
        graph.replay()
        ctx.adamw_step(other, float(torch.tensor(1e-2)), k, grad_scale=0.375, rounding="stochastic", seed=11)
    assert int(step) == 7
    for k in ("param", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale"):
        assert same(torch, a[k], b[k]), k
    scale.fill_(float("inf"))
    old = before(a)
    graph.replay()
    assert all(same(torch, a[k], old[k]) for k in ("param", "exp_avg", "exp_avg_sq", "avg_scale"))
    import paper_2512_11280_b200 as adasd
    assert ctx.status() == adasd.STATUS_NAN and ctx.status() == 0


def test_another_stream_and_twice_the_same(torch, ctx):
    g = torch.Generator(device="cuda").manual_seed(8)
    a, _ = tensor(torch, 500000, g, "bfloat16", "bfloat16", 8)
    b = before(a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ctx.adamw_step(ctx.adamw_table([a]), **OPT)
    ctx.adamw_step(ctx.adamw_table([b]), **OPT)
    torch.cuda.synchronize()
    assert all(same(torch, a[k], b[k]) for k in ("param", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale"))


def test_tables_that_are_refused(torch, ctx):
    import paper_2512_11280_b200 as adasd
    g = torch.Generator(device="cuda").manual_seed(9)
    t, _ = tensor(torch, 600, g, copy=True)
    e, _ = tensor(torch, 600, g, bits=8)

    def refused(code, *tensors):
        with pytest.raises(adasd.AdasdError) as err:
            ctx.adamw_table(list(tensors))
        assert err.value.code == code
    refused(adasd.ERR_SHAPE, t, t)                                            # the same tensor twice
    refused(adasd.ERR_SHAPE, t, dict(e, grad=t["param"][:600]))               # one array in two places
    refused(adasd.ERR_SHAPE, dict(t, grad=t["grad"][:599]))
    refused(adasd.ERR_SHAPE, dict(t, exp_avg=torch.zeros(1200, device="cuda")[::2]))
    refused(adasd.ERR_SHAPE, dict(e, avg_scale=e["avg_scale"][:2]))
    refused(adasd.ERR_DTYPE, dict(t, param=t["param"].half()))
    refused(adasd.ERR_DTYPE, dict(t, exp_avg_sq=t["exp_avg_sq"].bfloat16()))
    refused(adasd.ERR_DTYPE, dict(e, exp_avg_sq=e["exp_avg"]))
    refused(adasd.ERR_DTYPE, dict(t, param_copy=t["param"].clone()))
    refused(adasd.ERR_DEVICE, dict(t, grad=t["grad"].cpu()))
    with pytest.raises(adasd.AdasdError) as err:
        ctx.adamw_step(ctx.adamw_table([e]), **OPT, rounding="up")
    assert err.value.code == adasd.ERR_DTYPE
    with pytest.raises(adasd.AdasdError) as err:
        ctx.adamw_step(ctx.adamw_table([e]), **dict(OPT, step=0))
    assert err.value.code == adasd.ERR_SHAPE
