"""The text of a failed CUDA step (no GPU): what the step itself said of it comes through, as that of a tensor map that cannot be made."""
import os
import subprocess

from paper_2605_02218_b200 import build

PROGRAM = r"""
#include <cstdio>

#include "host.cuh"
using namespace covspec;
int main() {
  int st = status_of("attention", [] { g_cuda_error = "cuTensorMapEncodeTiled failed with code 1"; return cudaErrorInvalidValue; });
  printf("%d %s\n", st, g_cuda_error.c_str());
  st = status_of("attention", [] { return cudaSuccess; });
  printf("%d %s\n", st, g_cuda_error.c_str());
  st = status_of("attention", [] { return cudaErrorInvalidValue; });
  printf("%d %s\n", st, g_cuda_error.c_str());
}
"""


def test_a_step_that_says_what_failed_is_quoted(tmp_path):
    source, program = tmp_path / "errors.cu", tmp_path / "errors"
    source.write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-o", str(program), str(source)], check=True)
    said = subprocess.run([str(program)], capture_output=True, text=True, check=True).stdout.splitlines()
    assert said == ["-5 cuTensorMapEncodeTiled failed with code 1", "0 cuTensorMapEncodeTiled failed with code 1",
                    "-5 attention: invalid argument"]
