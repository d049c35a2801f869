"""Shared memory of another CTA may be written only once that CTA runs, and a CTA of a cluster may start later than the others:
every kernel waits at a barrier of its cluster first.  A kernel that does not is right in nearly every run."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = sorted(glob.glob(os.path.join(ROOT, "paper_2512_11280_b200", "csrc", "*.cuh")))
REMOTE = r"map_shared_rank\(|mapa_u32\(|cluster_allreduce<"
BARRIER = r"(?:cluster|this_cluster\(\))\.(?:sync|barrier_wait)\(\)|barrier\.cluster\.wait"


def kernels(path):
    """(name, text) of the kernels of a file, without comments."""
    text = re.sub(r"//[^\n]*", "", open(path).read())
    for part in re.split(r"__global__", text)[1:]:
        yield re.search(r"\w+_kernel\w*(?=\()", part).group(), part[: part.find("\n}\n")]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_a_cluster_barrier_stands_ahead_of_the_first_use_of_remote_shared_memory(path):
    for name, body in kernels(path):
        remote = re.search(REMOTE, body)
        if remote:
            assert re.search(BARRIER, body[: remote.start()]), name


def test_the_rule_sees_the_kernels_it_is_about():
    found = {name for path in FILES for name, body in kernels(path) if re.search(REMOTE, body)}
    assert {"score_kernel", "score_stream_kernel", "score_deep_kernel", "score_forward_kernel", "pref_pair_kernel", "static_vanilla_kernel"} <= found, found
