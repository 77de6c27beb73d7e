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
