"""Tensor maps of the head calls: the device is handed, and fetches, none that was not encoded for the call."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_11280_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_no_map_is_left_uninitialised():
    """A map that only some calls encode is zeros in the others, not what the stack held."""
    seen = 0
    for line in re.findall(r"^\s*CUtensorMap [^*;()]*;", source("adasd_head.cu"), re.M):
        for name in line.strip()[len("CUtensorMap "):-1].split(","):
            seen += 1
            assert "=" in name or name.strip().endswith("{}"), line
    assert seen >= 4


def test_maps_that_a_launch_may_lack_are_not_fetched():
    """The products of both gradients write grad_hidden by way of the sums: their map of what is stored is that of grad_weight, and there is
    none where that is not wanted."""
    found = re.findall(r"^([^\n]*)tma_prefetch\(&p\.out\);", source("adasd_head.cuh"), re.M)
    assert found
    for condition in found:
        assert "TILE_G " in condition and "want_w" in condition, condition
