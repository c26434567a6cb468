"""Host code of the paged key/value cache that needs no GPU: compiled by itself, with the CUDA calls it makes replaced."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")


def compiled_and_run(tmp_path, source):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists(os.path.join(CUDA, "include", "cuda_runtime.h")):
        pytest.skip("needs g++ and the CUDA headers")
    (tmp_path / "t.cpp").write_text(source)
    subprocess.run([gxx, "-std=c++17", "-O1", "-I", os.path.join(CUDA, "include"), "-I", os.path.join(ROOT, "paper_2508_18736_b200", "csrc"),
                    "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    return subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)


def test_the_current_device_is_put_back(tmp_path):
    got = compiled_and_run(tmp_path, r'''
#include <cstdio>
#include "kv.cuh"
static int current = 3, sets = 0;
static bool refuse = false;
extern "C" cudaError_t CUDARTAPI cudaGetDevice(int *d) { *d = current; return cudaSuccess; }
extern "C" cudaError_t CUDARTAPI cudaSetDevice(int d) { ++sets; if (refuse) return cudaErrorInvalidDevice; current = d; return cudaSuccess; }
int main() {
    { siso::OnDevice on(1); printf("%d %d ", current, on.error()); }
    printf("%d %d\n", current, sets);
    { siso::OnDevice on(3); printf("%d %d ", current, on.error()); }
    printf("%d %d\n", current, sets);
    refuse = true;
    { siso::OnDevice on(9); printf("%d %d ", current, on.error() != cudaSuccess); }
    printf("%d %d\n", current, sets);
}
''')
    assert got.returncode == 0 and got.stdout.splitlines() == ["1 0 3 2", "3 0 3 2", "3 1 3 3"], got.stdout + got.stderr
