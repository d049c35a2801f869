"""Head calls refuse arrays that they write where these overlap with what they read, or with one another."""
import itertools

import pytest
import torch

import paper_2512_11280_b200 as adasd
from tests.test_head_cpu import CTX

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the calls go on to look at the context, and there is none here")
N, D = 100, 64
# (never dereferenced: what overlaps is refused on the host, and what does not gets no further than the check for a device, or the context's kind)
AT = {name: 0x100000 * (k + 1) for k, name in enumerate(
    "hidden weight tok scratch logp entropy lse row_weight row_loss loss dl dH grad_hidden grad_weight".split())}
BYTES = dict(hidden=N * D * 2, scratch=4096, grad_hidden=N * D * 2, loss=4)


def logprob(a):
    return adasd.adasd_head_logprob(CTX, a["hidden"], D, a["weight"], D, D, a["tok"], N, a["scratch"], 4096, a["logp"], a["entropy"], a["lse"], None)


def grad(a):
    return adasd.adasd_head_logprob_grad(CTX, a["hidden"], D, a["weight"], D, D, a["tok"], N, a["lse"], a["entropy"], a["dl"], a["dH"], a["scratch"], 4096,
                                         a["grad_hidden"], D, a["grad_weight"], D, None)


def entropy(a):
    return adasd.adasd_head_cross_entropy(CTX, a["hidden"], D, a["weight"], D, D, a["tok"], N, a["row_weight"], adasd.CrossEntropyOptions(0.0, 0.0, 1.0),
                                          a["scratch"], 4096, a["row_loss"], a["loss"], a["logp"], a["lse"], a["grad_hidden"], D, a["grad_weight"], D, None)


# (the weight's extent, which hangs on the context's vocabulary, is tested with a device)
CALLS = [(logprob, "scratch logp entropy lse", "hidden tok"), (grad, "scratch grad_hidden", "hidden tok lse entropy dl dH"),
         (entropy, "scratch row_loss loss logp lse grad_hidden", "hidden tok row_weight")]


@pytest.mark.parametrize("call,written,read", CALLS)
def test_what_is_written_overlaps_with_nothing(call, written, read):
    assert call(AT) not in (adasd.ERR_SHAPE, adasd.ERR_ALIGN, adasd.ERR_NULL, 0)
    size = lambda name: BYTES.get(name, 4 * N)  # noqa: E731
    written, read = written.split(), read.split()
    pairs = list(itertools.combinations(written, 2)) + list(itertools.product(written, read))
    for a, b in pairs:
        # the same place; the last 16 bytes (4 of a single value) of one and the first of the other; next to one another is fine
        tail = 4 if "loss" in (a, b) else 16
        for at, refused in ((AT[b], True), (AT[b] + size(b) - tail, True), (AT[b] - size(a) + tail, True), (AT[b] + (size(b) + 15) // 16 * 16, False)):
            if a == "scratch" and at % 16:
                continue
            rc = call({**AT, a: at})
            assert (rc == adasd.ERR_SHAPE) == refused, (a, b, hex(at), rc)


def test_arrays_that_are_read_may_be_the_same():
    rc = grad({**AT, "entropy": AT["lse"], "dH": AT["dl"]})
    assert rc not in (adasd.ERR_SHAPE, 0)


# hidden states and their gradient as columns of one array: offset (elements) of the gradient, stride, and whether that overlaps
@pytest.mark.parametrize("first,stride,overlap", [(D, 2 * D, False), (D + 8, 2 * D + 8, False), (D - 1, 2 * D, True), (D + 1, 2 * D, True), (-D, 2 * D, False),
                                                  (-D + 1, 2 * D, True), (5 * 2 * D + D, 2 * D, False), (5 * 2 * D, 2 * D, True), (-7 * 2 * D - D, 2 * D, False),
                                                  (D, 2 * D - 1, True), (0, 2 * D, True), (N * 2 * D, 2 * D, False)])
def test_columns_of_one_array(first, stride, overlap):
    for call in ("grad", "entropy"):
        a = {**AT, "grad_hidden": AT["hidden"] + 2 * first}
        if call == "grad":
            rc = adasd.adasd_head_logprob_grad(CTX, a["hidden"], stride, a["weight"], D, D, a["tok"], N, a["lse"], None, a["dl"], None, a["scratch"], 4096,
                                               a["grad_hidden"], stride, None, 0, None)
        else:
            rc = adasd.adasd_head_cross_entropy(CTX, a["hidden"], stride, a["weight"], D, D, a["tok"], N, None, adasd.CrossEntropyOptions(0.0, 0.0, 1.0),
                                                a["scratch"], 4096, a["row_loss"], None, None, None, a["grad_hidden"], stride, None, 0, None)
        assert (rc == adasd.ERR_SHAPE) == overlap, (call, rc)


def test_rows_with_other_strides_overlap():
    a = {**AT, "grad_hidden": AT["hidden"] + 2 * D}
    rc = adasd.adasd_head_logprob_grad(CTX, a["hidden"], 2 * D, a["weight"], D, D, a["tok"], N, a["lse"], None, a["dl"], None, a["scratch"], 4096,
                                       a["grad_hidden"], 2 * D + 2, None, 0, None)
    assert rc == adasd.ERR_SHAPE
