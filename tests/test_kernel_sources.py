"""Rules of the CUDA programming model that no run shows to be broken, read off the
kernels' sources (comments left out)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2608_08340_gb300", "csrc")
SOURCES = sorted(n for n in os.listdir(CSRC) if n.endswith((".cu", ".cuh")))


def _code(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def test_there_are_sources():
    assert "distill.cu" in SOURCES and "embed.cu" in SOURCES


@pytest.mark.parametrize("name", SOURCES)
def test_a_peers_shared_memory_is_touched_behind_a_cluster_barrier(name):
    """Blocks of a cluster run together, but only a barrier of the cluster tells that
    a peer has begun: before it, its shared memory is not there to be accessed."""
    for kernel in re.split(r"__global__", _code(name))[1:]:
        first = kernel.find("map_shared_rank(")
        if first >= 0:
            assert re.search(r"cluster\.(sync|barrier_wait)\(", kernel[:first]), name


@pytest.mark.parametrize("name", SOURCES)
def test_shared_arrays_of_small_values_state_their_alignment(name):
    """An array of 1- or 2-byte values lies on any such boundary unless it says
    otherwise, and the kernels clear and copy such arrays in words."""
    small = r"(u?int(8|16)_t|(unsigned\s+|signed\s+)?(short|char)|__half|__nv_bfloat16)"
    found = re.findall(rf"__shared__\s+{small}\s+\w+\s*\[", _code(name))
    assert not found, name
