"""Instructions that a warp has to reach as one, by reading: in routing's lists, the 8-bit products and sampling the lanes of a warp
are brought together in front of every cluster barrier, and in front of each read of tensor memory."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_07008_b200", "csrc")


def statements(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    return [s.strip() for s in re.split(r"[;{}]", text) if s.strip()]


@pytest.mark.parametrize("name", ["rk_experts.cu", "rk_matmul8.cu", "rk_sample.cu"])
def test_cluster_barriers_bring_the_warp_together(name):
    code = statements(name)
    barriers = [i for i, s in enumerate(code) if s in ("cluster_arrive()", "cluster_wait()")]
    assert barriers and "barrier.cluster" not in "".join(code)
    for i in barriers:
        assert code[i - 1] == "__syncwarp()" or (code[i] == "cluster_wait()" and code[i - 1] == "cluster_arrive()"), code[i - 2:i + 1]


def test_the_8_bit_products_read_tensor_memory_with_whole_warps():
    code = statements("rk_matmul8.cu")
    loads = [i for i, s in enumerate(code) if s.startswith("tmem_ld_")]
    assert loads and all(code[i - 1] == "__syncwarp()" for i in loads)
