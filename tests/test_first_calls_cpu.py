"""Threads whose first calls meet (ctypes lets them): the per-process look-ups of the launchers, with the CUDA runtime's entry points
replaced by slow ones, on the CPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cuda_runtime.h>
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>

static void pause() { std::this_thread::sleep_for(std::chrono::milliseconds(100)); }
static std::atomic<int> attributes{0};
static cudaError_t slow_entry(const char*, void** p, unsigned long long, cudaDriverEntryPointQueryResult* r) {
  pause();
  *p = (void*)0x1000;
  *r = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
static cudaError_t one_device(int* d) { *d = 3; return cudaSuccess; }
template <typename K> static cudaError_t slow_attribute(K, cudaFuncAttribute, int) { pause(); ++attributes; return cudaSuccess; }
static cudaError_t count_sms(int* n, cudaDeviceAttr, int) { *n = 148; return cudaSuccess; }
#define cudaGetDriverEntryPoint slow_entry
#define cudaGetDevice one_device
#define cudaFuncSetAttribute slow_attribute
#define cudaDeviceGetAttribute count_sms
#include "tc_common.cuh"

namespace pbt { bool serial_launches() { return true; } }

int main() {
  std::atomic<int> no_function{0}, not_set_up{0};
  static pbt::tc::DeviceSetup setup;
  std::vector<std::thread> threads;
  for (int i = 0; i < 8; ++i)
    threads.emplace_back([&, i] {
      std::this_thread::sleep_for(std::chrono::milliseconds(10 * i));       // some while the first one looks up
      if (pbt::tc::encode_fn() == nullptr) ++no_function;
      int sms = 0;
      if (pbt::tc::device_setup(&setup, 0, 1000, &sms) != cudaSuccess || sms != 148 || attributes == 0) ++not_set_up;
    });
  for (auto& t : threads) t.join();
  const int before = attributes;
  int sms = 0;
  pbt::tc::device_setup(&setup, 0, 1000, &sms);
  printf("%d %d %d %d\n", no_function.load(), not_set_up.load(), attributes.load() - before, sms);
}
'''


def test_first_calls_of_several_threads_all_find_the_driver_entry_point(tmp_path):
    from paper_1711_09846_b200 import build
    source, program = tmp_path / "first_calls.cu", tmp_path / "first_calls"
    source.write_text(SOURCE)
    flags = [f for f in build.NVCC_FLAGS if f not in ("-O3", "-lineinfo")]
    subprocess.run([build._nvcc(), *flags, str(source), "-o", str(program)], check=True, capture_output=True)
    out = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [0, 0, 0, 148]
