"""What the launch helpers of csrc/kernels.h hand to the runtime (no GPU needed: the launch itself is a stand-in)."""
import os
import shutil
import subprocess

import pytest

from test_kv8_refusals import ROOT

SOURCE = r"""
#include <stdio.h>
#include "kernels.h"
extern "C" cudaError_t CUDARTAPI cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void** args) {
  printf("%u %u %u  %u %u %u  %zu %d\n", c->gridDim.x, c->gridDim.y, c->gridDim.z, c->blockDim.x, c->blockDim.y, c->blockDim.z, c->dynamicSmemBytes,
         *static_cast<int*>(args[0]));
  return cudaSuccess;
}
__global__ void kernel(int) {}
int main() {
  dart::launch_pdl(kernel, dim3(2, 3, 4), dim3(32, 4, 2), 100, nullptr, 7);
  dart::launch_ahead(kernel, dim3(5), dim3(8, 16), 0, nullptr, 8);
  dart::launch_ahead(kernel, dim3(6), 256, 0, nullptr, 9);
}
"""


def test_blocks_of_more_than_one_dimension_are_launched_whole(tmp_path):
    nvcc = os.environ.get("NVCC", "nvcc")
    if shutil.which(nvcc) is None:
        pytest.skip("needs nvcc")
    src, exe = tmp_path / "launch.cu", tmp_path / "launch"
    src.write_text(SOURCE)
    subprocess.check_call([nvcc, "-std=c++17", "-cudart", "shared", "-gencode", "arch=compute_100a,code=sm_100a", "-I",
                           os.path.join(ROOT, "paper_2601_19278_b200", "csrc"), str(src), "-o", str(exe)])
    got = [line.split() for line in subprocess.check_output([str(exe)], text=True).splitlines()]
    assert got == ["2 3 4 32 4 2 100 7".split(), "5 1 1 8 16 1 0 8".split(), "6 1 1 256 1 1 0 9".split()]
