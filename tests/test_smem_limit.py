"""The limit of a kernel's dynamic shared memory, set by two threads at once (no device: the runtime's two calls are stood in for)."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# The larger limit's call waits, once the attribute has its value, for the smaller one's (300 ms at most): without an order between threads
# the smaller value lands on top, and the larger one is remembered.
HARNESS = """
#include <cuda_runtime.h>
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
static std::atomic<int> attribute{0}, small_started{0}, large_set{0}, small_done{0}, calls{0};
template <typename F> static bool within(F f, int ms) {
  for (auto t0 = std::chrono::steady_clock::now(); std::chrono::steady_clock::now() - t0 < std::chrono::milliseconds(ms);)
    if (f()) return true;
  return f();
}
static cudaError_t stand_in_device(int* dev) { *dev = 3; return cudaSuccess; }
template <typename K> static cudaError_t stand_in_set(K, cudaFuncAttribute, int bytes) {
  ++calls;
  if (bytes == 1000) {
    within([] { return small_started.load() != 0; }, 300);
    attribute = bytes;
    large_set = 1;
    within([] { return small_done.load() != 0; }, 300);
  } else {
    small_started = 1;
    within([] { return large_set.load() != 0; }, 300);
    attribute = bytes;
  }
  return cudaSuccess;
}
#define cudaGetDevice stand_in_device
#define cudaFuncSetAttribute stand_in_set
#include "common.cuh"
static void kernel() {}
int main() {
  bsr::SmemLimit lim;
  std::thread large([&] { bsr::ensure_smem(lim, kernel, 1000); });
  std::thread small([&] { bsr::ensure_smem(lim, kernel, 200); small_done = 1; });
  large.join();
  small.join();
  if (!bsr::ensure_smem(lim, kernel, 1000) || attribute < 1000) return std::printf("the limit is %d, 1000 were asked for\\n", attribute.load()), 1;
  const int before = calls;
  if (!bsr::ensure_smem(lim, kernel, 900) || calls != before) return std::printf("asked again\\n"), 1;
  return std::printf("fine\\n"), 0;
}
"""


def test_two_threads_leave_the_larger_limit(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    src, exe = tmp_path / "harness.cu", tmp_path / "harness"
    src.write_text(HARNESS)
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "paper_2405_10951_b200", "csrc"), "-o", str(exe), str(src)], check=True, capture_output=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout == "fine\n", run.stdout + run.stderr
