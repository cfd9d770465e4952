"""Instructions that a warp has to reach as one, by reading: the cluster barriers of every kernel go through two wrappers, which
bring the warp's lanes together first, and the 8-bit products do so in front of each read of tensor memory."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_07008_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_cluster_barriers_bring_the_warp_together():
    ptx = source("rk_ptx.cuh")
    for name in ("arrive", "wait"):
        body = re.search(r"void cluster_%s\(\) \{(.*?)\n\}" % name, ptx, flags=re.S).group(1)
        assert "barrier.cluster." + name in body
        assert body.strip().startswith("__syncwarp();")
    assert ptx.count("barrier.cluster.") == 2
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        assert "barrier.cluster." not in source(os.path.basename(path)), path


def test_the_8_bit_products_read_tensor_memory_with_whole_warps():
    loads = re.findall(r"([^\n;]*;)\s*tmem_ld_x32\(", source("rk_matmul8.cu"))
    assert loads and all("__syncwarp();" in before for before in loads)
