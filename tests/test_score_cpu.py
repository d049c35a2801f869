"""Refusals of the scoring and loss calls that need no GPU: null contexts, options out of range, which are looked at before anything
of a context or a device is."""
import ctypes
import math

import pytest

import paper_2512_11280_b200 as adasd

P = 0x10000          # never dereferenced: every case below is refused on the host


@pytest.fixture(scope="module")
def ctx():
    return ctypes.addressof(_BLOCK)


_BLOCK = ctypes.create_string_buffer(1 << 16)       # stands for a context that no call gets as far as


def policy(ctx, adv=P, ref=P, rl=P, kl=None, n=4, options=True, **o):
    o = adasd.PolicyOptions(*{**dict(clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, scale=1.0), **o}.values())
    return adasd.adasd_policy_loss(ctx, P, 100, P, n, adv, None, ref, None, o if options else None, rl, None, None, None, kl, None, 0, None)


def preference(ctx, start=P, scratch=P, seq=P, loss=P, n=4, pairs=2, options=True, **o):
    o = adasd.PreferenceOptions(*{**dict(rule=0, average=0, beta=0.1, margin=0.0, label_smoothing=0.0, scale=1.0), **o}.values())
    return adasd.adasd_preference_loss(ctx, P, 100, P, n, start, pairs, None, None, o if options else None, scratch, seq, loss, None, None, 0, None)


def test_null_arguments(ctx):
    assert adasd.adasd_token_logprob(None, P, 100, P, 4, P, None, None, None) == adasd.ERR_NULL
    assert adasd.adasd_token_logprob(ctx, P, 100, P, 4, None, None, None, None) == adasd.ERR_NULL
    assert adasd.adasd_token_logprob(ctx, None, 100, P, 4, P, None, None, None) == adasd.ERR_NULL
    assert adasd.adasd_token_logprob(ctx, P, 100, None, 4, P, None, None, None) == adasd.ERR_NULL
    assert adasd.adasd_token_logprob_grad(None, P, 100, P, 4, P, None, P, 100, None) == adasd.ERR_NULL
    assert adasd.adasd_token_logprob_grad(ctx, P, 100, P, 4, None, None, P, 100, None) == adasd.ERR_NULL
    assert adasd.adasd_token_logprob_grad(ctx, P, 100, P, 4, P, None, None, 100, None) == adasd.ERR_NULL
    assert policy(None) == adasd.ERR_NULL and preference(None) == adasd.ERR_NULL
    assert policy(ctx, options=False) == adasd.ERR_NULL and preference(ctx, options=False) == adasd.ERR_NULL
    assert policy(ctx, adv=None) == adasd.ERR_NULL and policy(ctx, rl=None) == adasd.ERR_NULL
    assert policy(ctx, ref=None, kl_coef=0.1) == adasd.ERR_NULL and policy(ctx, ref=None, kl=P) == adasd.ERR_NULL
    for name in ("start", "scratch", "seq", "loss"):
        assert preference(ctx, **{name: None}) == adasd.ERR_NULL, name


@pytest.mark.parametrize("name,bad", [("clip_low", (-0.1, 1.5, math.nan, math.inf)), ("clip_high", (-0.1, math.nan, math.inf)),
                                      ("kl_coef", (-1.0, math.nan, math.inf)), ("entropy_coef", (math.nan, math.inf)),
                                      ("scale", (math.nan, math.inf))])
def test_policy_options(ctx, name, bad):
    for v in bad:
        assert policy(ctx, **{name: v}) == adasd.ERR_SHAPE, v


@pytest.mark.parametrize("name,bad,code", [("rule", (-1, 3), adasd.ERR_DTYPE), ("average", (-1, 2), adasd.ERR_DTYPE),
                                           ("beta", (0.0, -1.0, math.nan, math.inf), adasd.ERR_SHAPE), ("margin", (math.nan,), adasd.ERR_SHAPE),
                                           ("label_smoothing", (-0.1, 0.6, math.nan), adasd.ERR_SHAPE), ("scale", (math.inf,), adasd.ERR_SHAPE),
                                           ("pairs", (-1, 1 << 28), adasd.ERR_SHAPE)])
def test_preference_options(ctx, name, bad, code):
    for v in bad:
        assert preference(ctx, **{name: v}) == code, v
    for rule in (adasd.PREF_SQUARED, adasd.PREF_HINGE):
        assert preference(ctx, rule=rule, label_smoothing=0.1) == adasd.ERR_SHAPE


def test_sizes_of_the_header_match_the_binding():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "adasd.h")).read()
    got = dict(re.findall(r"#define ADASD_(PREF_[A-Z_]+) (\d+)", text))
    assert {k: int(v) for k, v in got.items()} == {"PREF_SIGMOID": adasd.PREF_SIGMOID, "PREF_SQUARED": adasd.PREF_SQUARED,
                                                   "PREF_HINGE": adasd.PREF_HINGE, "PREF_SCRATCH_PER_ROW": adasd.PREF_SCRATCH_PER_ROW}
