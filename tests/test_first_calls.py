"""First calls from several host threads, on the host: the lookup of the driver's tensor-map encoder is stood in for by a slow one."""
import os
import subprocess

from paper_2609_01024_b200 import build

SOURCE = r"""
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <chrono>
#include <thread>

static std::atomic<int> lookups{0};
static cudaError_t slow_lookup(const char *, void **sym, unsigned long long, cudaDriverEntryPointQueryResult *result) {
  ++lookups;
  std::this_thread::sleep_for(std::chrono::milliseconds(400));
  *sym = (void *)&lookups;
  *result = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
#undef cudaGetDriverEntryPoint
#define cudaGetDriverEntryPoint slow_lookup
#include "tc_ptx.cuh"

int main() {
  bool first = false, second = false;
  std::thread a([&] { first = pcomoe::encode_fn() != nullptr; });
  std::this_thread::sleep_for(std::chrono::milliseconds(100));
  std::thread b([&] { second = pcomoe::encode_fn() != nullptr; });
  a.join();
  b.join();
  return (first ? 0 : 1) + (second ? 0 : 2) + (lookups == 1 ? 0 : 4);
}
"""


def test_a_second_thread_waits_for_the_first_ones_lookup(tmp_path):
    """A valid call while another thread makes the first one must not find 'tried, and nothing there'."""
    src, exe = tmp_path / "lookup.cu", tmp_path / "lookup"
    src.write_text(SOURCE)
    subprocess.run([build.NVCC, *build.FLAGS, str(src), "-o", str(exe), "-lcudart"], check=True, capture_output=True)
    env = dict(os.environ, LD_LIBRARY_PATH="/usr/local/cuda/lib64:" + os.environ.get("LD_LIBRARY_PATH", ""))
    assert subprocess.run([str(exe)], env=env).returncode == 0
