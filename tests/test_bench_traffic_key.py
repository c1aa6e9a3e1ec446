"""The recorded DRAM traffic of the expert GEMMs belongs to the sources that decide it."""
import os
import shutil

import bench


def _copy(tmp_path):
    dst = tmp_path / "csrc"
    shutil.copytree(bench.CSRC, dst)
    return str(dst)


def test_every_source_that_decides_the_traffic_is_in_the_key(tmp_path):
    csrc = _copy(tmp_path)
    key = bench._src_hash(csrc=csrc)
    assert key == bench._src_hash()
    # the kernel, its launches (tiles, rings, rules), what their code includes
    for name in ("gemm_tc.cu", "gemm_tc_kernel.cuh", "gemm_tc.h", "common.cuh", "launch.h", "act.cuh",
                 "philox.cuh"):
        path = os.path.join(csrc, name)
        text = open(path).read()
        open(path, "w").write(text + "\n// changed\n")
        assert bench._src_hash(csrc=csrc) != key, name
        open(path, "w").write(text)
    assert bench._src_hash(csrc=csrc) == key


def test_sources_of_other_kernels_are_not(tmp_path):
    csrc = _copy(tmp_path)
    key = bench._src_hash(csrc=csrc)
    for name in ("balance.cu", "linear_tile.cuh", "route.cu", "ecmoe_api.cu"):
        open(os.path.join(csrc, name), "a").write("\n// changed\n")
    assert bench._src_hash(csrc=csrc) == key
