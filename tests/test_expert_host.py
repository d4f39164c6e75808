"""Host side of the expert operators against a stand-in for the CUDA runtime: no GPU needed."""
import os
import subprocess

import pytest

from paper_2111_00153_b200 import build as B

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "sort_clusters.cpp")


@pytest.fixture(scope="module")
def sort_clusters(tmp_path_factory):
    d = tmp_path_factory.mktemp("native")
    nvcc = B._nvcc()
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    # (the device code is compiled because it is in the same file, as fast as it can be: nothing of it is run)
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-Xptxas", "-O0", "-c", os.path.join(B.CSRC, "expert.cu"), "-o", str(d / "expert.o")])
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", include, SOURCE, str(d / "expert.o"), "-o", str(d / "sort_clusters"), "-pthread"])
    return str(d / "sort_clusters")


@pytest.mark.parametrize("device, sixteen, eight", [("slow", 4, 0), ("never", 0, 3), ("no_room", 0, 3)])
def test_clusters_of_the_sort(sort_clusters, device, sixteen, eight):
    """Threads that sort for the first time together all get sixteen CTAs; where there are none of sixteen, no launch finds that out by being refused."""
    out = subprocess.check_output([sort_clusters, device], text=True, timeout=60)
    assert out.split() == ["0", str(sixteen), str(eight)]
