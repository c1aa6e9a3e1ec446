"""Kernel attributes are set once for every device of a process, not once for the process (CPU: the helper
that the launches use, compiled with a stand-in for the current device)."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2604_01622_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "launch.h"
static int current = 0;
extern "C" cudaError_t cudaGetDevice(int* d) { *d = current; return cudaSuccess; }
int main() {
  ecmoe::PerDevice once;
  int made[100] = {0}, fail = 0;
  auto ask = [&](int dev) {
    current = dev;
    int v = 0;
    const cudaError_t e = once.get(&v, [&](int* out) {
      ++made[dev];
      *out = 10 + dev;
      return fail ? cudaErrorNotSupported : cudaSuccess;
    });
    return e == cudaSuccess ? v : -1;
  };
  std::printf("%d %d %d %d ", ask(0), ask(0), ask(1), ask(0));
  fail = 1;
  std::printf("%d ", ask(2));
  fail = 0;
  std::printf("%d %d %d %d ", ask(2), ask(2), ask(99), ask(99));
  std::printf("%d %d %d %d\n", made[0], made[1], made[2], made[99]);
}
"""


def test_once_for_every_device(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    if not os.path.exists(os.path.join(inc, "cuda_runtime.h")):
        pytest.skip("no CUDA headers")
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-I", inc, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    # devices 0, 0, 1, 0; a failure is asked again; past the table every time
    assert out[:9] == ["10", "10", "11", "10", "-1", "12", "12", "109", "109"]
    assert out[9:] == ["1", "1", "2", "2"]


def test_launches_latch_nothing_for_the_whole_process():
    """Dynamic shared memory is asked for on every call or through the helper."""
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for at in re.finditer(r"cudaFuncSetAttribute", text):
            before = text[max(0, at.start() - 600):at.start()]
            assert not re.search(r"static (bool|int) \w+ = (false|0);", before), name
