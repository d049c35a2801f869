"""Refusals of the head calls that need no GPU."""
import ctypes
import math

import pytest

import paper_2512_11280_b200 as adasd

P = 0x10000          # never dereferenced: every case below is refused on the host
_BLOCK = ctypes.create_string_buffer(1 << 16)       # stands for a context that no call gets as far as
CTX = ctypes.addressof(_BLOCK)
SHARED = dict(hidden=P, hs=64, weight=P, ws=64, dim=64, tok=P, n=4, scratch=P, bytes=1 << 40)


def logprob(ctx=CTX, lp=P, H=None, lse=None, **o):
    a = {**SHARED, **o}
    return adasd.adasd_head_logprob(ctx, a["hidden"], a["hs"], a["weight"], a["ws"], a["dim"], a["tok"], a["n"], a["scratch"], a["bytes"], lp, H, lse, None)


def grad(ctx=CTX, lse=P, ent=None, dl=P, dH=None, gh=P, ghs=64, gw=None, gws=64, **o):
    a = {**SHARED, **o}
    return adasd.adasd_head_logprob_grad(ctx, a["hidden"], a["hs"], a["weight"], a["ws"], a["dim"], a["tok"], a["n"], lse, ent, dl, dH, a["scratch"],
                                         a["bytes"], gh, ghs, gw, gws, None)


def entropy(ctx=CTX, rw=None, rl=P, loss=None, options=True, e=0.0, c=0.0, scale=1.0, gh=None, ghs=64, gw=None, gws=64, **o):
    a = {**SHARED, **o}
    return adasd.adasd_head_cross_entropy(ctx, a["hidden"], a["hs"], a["weight"], a["ws"], a["dim"], a["tok"], a["n"], rw,
                                          adasd.CrossEntropyOptions(e, c, scale) if options else None, a["scratch"], a["bytes"], rl, loss, None, None,
                                          gh, ghs, gw, gws, None)


def test_null_arguments():
    assert logprob(ctx=None) == adasd.ERR_NULL and logprob(lp=None) == adasd.ERR_NULL
    assert grad(ctx=None) == adasd.ERR_NULL and grad(lse=None) == adasd.ERR_NULL and grad(dl=None) == adasd.ERR_NULL
    assert grad(dH=P) == adasd.ERR_NULL and grad(gh=None) == adasd.ERR_NULL
    assert entropy(ctx=None) == adasd.ERR_NULL and entropy(rl=None) == adasd.ERR_NULL and entropy(options=False) == adasd.ERR_NULL
    for name in ("hidden", "weight", "tok", "scratch"):
        for call in (logprob, grad, entropy):
            assert call(**{name: None}) == adasd.ERR_NULL, name
    assert adasd.adasd_head_scratch(None, 1, 64, 0)[0] == adasd.ERR_NULL


@pytest.mark.parametrize("call", [logprob, grad, entropy])
def test_sizes_and_strides(call):
    for bad in (dict(n=-1), dict(n=(1 << 22) + 1), dict(dim=0), dict(dim=60), dict(dim=65544, hs=65544, ws=65544), dict(hs=63), dict(ws=56), dict(ws=68),
                dict(hs=(1 << 33) + 1), dict(ws=(1 << 33) + 8)):
        assert call(**bad) == adasd.ERR_SHAPE, bad
    for bad in (dict(hidden=P + 1), dict(weight=P + 8), dict(scratch=P + 8), dict(tok=P + 2)):
        assert call(**bad) == adasd.ERR_ALIGN, bad


@pytest.mark.parametrize("call", [grad, entropy])
def test_gradients(call):
    for bad in (dict(gh=P, ghs=63), dict(gh=P, gw=P, gws=56), dict(gh=P, gw=P, gws=68), dict(gh=P, ghs=(1 << 33) + 1)):
        assert call(**bad) == adasd.ERR_SHAPE, bad
    for bad in (dict(gh=P + 1), dict(gw=P + 8)):
        assert call(**bad) == adasd.ERR_ALIGN, bad


def test_options_and_arrays():
    for bad in (dict(e=-0.1), dict(e=1.0), dict(e=math.nan), dict(c=-1.0), dict(c=math.inf), dict(c=math.nan), dict(scale=math.inf)):
        assert entropy(**bad) == adasd.ERR_SHAPE, bad
    for bad in (dict(rw=P + 1), dict(rl=P + 2), dict(loss=P + 2)):
        assert entropy(**bad) == adasd.ERR_ALIGN, bad
    for bad in (dict(lp=P + 1), dict(H=P + 2), dict(lse=P + 2)):
        assert logprob(**bad) == adasd.ERR_ALIGN, bad
    for bad in (dict(lse=P + 1), dict(dl=P + 2), dict(ent=P, dH=P + 2), dict(ent=P + 1, dH=P)):
        assert grad(**bad) == adasd.ERR_ALIGN, bad


def test_scratch_sizes():
    for bad in ((-1, 64, 0), (1, 60, 0), (1, 0, 0), (1, 64, 2), ((1 << 22) + 1, 64, 0)):
        assert adasd.adasd_head_scratch(CTX, *bad)[0] == adasd.ERR_SHAPE, bad
