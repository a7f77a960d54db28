"""Host threads that raise one kernel's shared-memory limit to different sizes: afterwards the limit that is noted is
the one that is set.  The CUDA runtime is a fake of two functions that holds the larger size's call back until the
smaller one's has had its chance."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <thread>
#include "smem_limit.cuh"

static std::atomic<int> limit, sets, inside;
static constexpr int kLarge = 98304, kSmall = 49152;
extern "C" cudaError_t cudaGetDevice(int *d) { *d = 3; return cudaSuccess; }
extern "C" cudaError_t cudaFuncSetAttribute(const void *, cudaFuncAttribute, int bytes)
{
    limit = bytes;
    ++sets;
    if (bytes == kLarge) {
        inside = 1;                        // the smaller size may come now; wait for it, not for ever
        for (int i = 0; i < 300 && sets < 2; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
        std::this_thread::sleep_for(std::chrono::milliseconds(50));
    }
    return cudaSuccess;
}
static void kernel() {}
int main()
{
    static std::atomic<int> raised[w4a8::kMaxDevices];
    std::thread a([] { w4a8::raise_smem_limit(&kernel, kLarge, raised); });
    while (!inside) std::this_thread::yield();
    std::thread b([] { w4a8::raise_smem_limit(&kernel, kSmall, raised); });
    a.join();
    b.join();
    const int again = sets;
    w4a8::raise_smem_limit(&kernel, kSmall, raised);
    w4a8::raise_smem_limit(&kernel, kLarge, raised);
    std::printf("%d %d %d %d\n", limit.load(), raised[3].load(), sets.load(), again);
    return limit >= kLarge && raised[3] == limit ? 0 : 1;
}
"""


def test_two_threads_with_different_sizes(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", os.path.join(ROOT, "paper_2311_05161_b200", "csrc"), "-I",
                    os.path.join(CUDA, "include"), "-o", str(exe), str(src)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert got.returncode == 0, got.stdout
    assert got.stdout.split() == ["98304", "98304", "1", "1"]
