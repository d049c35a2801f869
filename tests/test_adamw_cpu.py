"""Refusals of the AdamW step that need no GPU."""
import ctypes
import math
import os
import re

import pytest

import paper_2512_11280_b200 as adasd

P = 0x10000          # never dereferenced: every case below is refused on the host
_BLOCK = ctypes.create_string_buffer(1 << 16)       # stands for a context that no call gets as far as


def call(ctx=True, n_tensors=1, table=True, options=True, tensor=(), **o):
    t = (adasd.AdamwTensor * 1)()
    values = dict(param=P, grad=P, exp_avg=P, exp_avg_sq=P, avg_scale=P, sq_scale=P, param_copy=None, n=10, weight_decay=0.0, param_dtype=adasd.ADASD_FP32,
                  grad_dtype=adasd.ADASD_BF16, state_bits=32)
    for k, v in {**values, **dict(tensor)}.items():
        setattr(t[0], k, v)
    opt = adasd.AdamwOptions(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1), **o})
    return adasd.adasd_adamw_step(ctypes.addressof(_BLOCK) if ctx else None, t if table else None, n_tensors, opt if options else None, None)


def test_null_arguments():
    assert call(ctx=False) == adasd.ERR_NULL and call(table=False) == adasd.ERR_NULL and call(options=False) == adasd.ERR_NULL
    for name in ("param", "grad", "exp_avg", "exp_avg_sq"):
        assert call(tensor={name: None}) == adasd.ERR_NULL, name
    for name in ("avg_scale", "sq_scale"):
        assert call(tensor={name: None, "state_bits": 8}) == adasd.ERR_NULL, name


@pytest.mark.parametrize("name,bad", [("lr", (math.nan, math.inf)), ("beta1", (-0.1, 1.0, math.nan)), ("beta2", (-0.1, 1.0, math.nan)),
                                      ("eps", (0.0, -1e-8, 1e-31, math.nan, math.inf)), ("grad_scale", (math.nan, math.inf)), ("step", (0, -3))])
def test_options(name, bad):
    for v in bad:
        assert call(**{name: v}) == adasd.ERR_SHAPE, v
    assert call(stochastic=2) == adasd.ERR_DTYPE
    for name in ("lr_dev", "grad_scale_dev", "step_dev"):
        assert call(**{name: P + 2}) == adasd.ERR_ALIGN
    assert call(n_tensors=-1) == adasd.ERR_SHAPE


def test_tensors():
    for bad in (dict(param_dtype=2), dict(grad_dtype=-1), dict(state_bits=16), dict(param_copy=P, param_dtype=adasd.ADASD_BF16)):
        assert call(tensor=bad) == adasd.ERR_DTYPE, bad
    for bad in (dict(n=-1), dict(n=(1 << 40) + 1), dict(weight_decay=math.nan)):
        assert call(tensor=bad) == adasd.ERR_SHAPE, bad
    for bad in (dict(param=P + 2), dict(grad=P + 1), dict(exp_avg=P + 2), dict(exp_avg_sq=P + 1), dict(param_copy=P + 1),
                dict(avg_scale=P + 1, state_bits=8), dict(sq_scale=P + 2, state_bits=8)):
        assert call(tensor=bad) == adasd.ERR_ALIGN, bad


def test_sizes_of_the_header_match_the_binding():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "adasd.h")).read()
    assert int(re.search(r"#define ADASD_ADAMW_BLOCK (\d+)", text).group(1)) == adasd.ADAMW_BLOCK
    # natural alignment in both: seven addresses, a length, four words; five doubles, three words (and four bytes), three addresses
    assert ctypes.sizeof(adasd.AdamwTensor) == 7 * 8 + 8 + 4 * 4 and ctypes.sizeof(adasd.AdamwOptions) == 5 * 8 + 16 + 3 * 8
