"""What a process's first calls set up holds for all threads that come meanwhile (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# The runtime's lookup of the driver's function that encodes tensor maps, as slow as a cold driver's, in place of the real one
SOURCE = r"""
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>
#include "xrl_umma.cuh"
static std::atomic<int> lookups{0};
extern "C" cudaError_t cudaGetDriverEntryPoint(const char*, void** fn, unsigned long long, cudaDriverEntryPointQueryResult* r) {
  lookups++;
  std::this_thread::sleep_for(std::chrono::milliseconds(100));
  static int place;
  *fn = &place;
  *r = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
int main() {
  std::vector<std::thread> threads;
  std::atomic<int> without{0};
  for (int i = 0; i < 8; ++i)
    threads.emplace_back([&, i] {
      std::this_thread::sleep_for(std::chrono::milliseconds(5 * i));
      if (!xrl::umma::encode_fn()) without++;
    });
  for (auto& t : threads) t.join();
  printf("%d threads without it, %d lookups\n", without.load(), lookups.load());
  return without.load() ? 1 : 0;
}
"""


def test_the_encoding_function_is_there_for_every_thread(tmp_path):
    from paper_2304_14698_b200 import build
    nvcc = build._nvcc()
    src, exe = tmp_path / "first.cu", tmp_path / "first"
    src.write_text(SOURCE)
    lib = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc") or nvcc))), "lib64")
    if not os.path.exists(os.path.join(lib, "libcudart.so")):
        pytest.skip("no shared runtime to put a function in front of")
    r = subprocess.run([nvcc, *build.NVCC_FLAGS, "-cudart", "shared", "-Xcompiler", "-pthread", str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, env={**os.environ, "LD_LIBRARY_PATH": lib}, timeout=60)
    assert r.returncode == 0 and "0 threads without it" in r.stdout, r.stdout + r.stderr
