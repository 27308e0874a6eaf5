"""First calls from several threads at once: what the library remembers per device is written without a data race (the compiler's
thread sanitizer over the headers' host code, with stand-ins for the CUDA calls)."""
import os
import shutil
import subprocess

import pytest

from paper_2504_05598_b200 import build

PROGRAM = r"""
#include <thread>
#include <vector>
#include "pages.cuh"
static void kernel(int) {}
int main() {
    static ClusterRoom room;
    static SmemAttrOnce attr;
    int got[4] = {};
    std::vector<std::thread> threads;
    for (int i = 0; i < 4; ++i)
        threads.emplace_back([&, i] {
            for (int r = 0; r < 200; ++r)
                got[i] = current_sms() + (attr.set(kernel, 1000) == cudaSuccess) + room.best(kernel, 256, 0, 8, 1 + r % 40);
        });
    for (auto &t : threads) t.join();
    for (int i = 0; i < 4; ++i)
        if (got[i] != 148 + 1 + 14) return 2;      // (40 steps, 8 clusters: of 14 CTAs, three steps each)
    return 0;
}
"""


STAND_INS = r"""
extern "C" int cudaGetDevice(int *d) { *d = 3; return 0; }
extern "C" int cudaDeviceGetAttribute(int *v, int, int) { *v = 148; return 0; }
extern "C" int cudaFuncSetAttribute(const void *, int, int) { return 0; }
extern "C" int cudaOccupancyMaxActiveClusters(int *n, const void *, const void *) { *n = 8; return 0; }
extern "C" int cudaGetLastError() { return 0; }
"""


@pytest.mark.skipif(shutil.which("nvcc") is None, reason="needs nvcc")
def test_first_calls_of_several_threads(tmp_path):
    (tmp_path / "first.cu").write_text(PROGRAM)
    (tmp_path / "calls.cpp").write_text(STAND_INS)
    exe = str(tmp_path / "first")
    made = subprocess.run(["nvcc", "-std=c++17", "-g", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "shared", "-Xcompiler", "-fsanitize=thread",
                           "-I", build.CSRC, str(tmp_path / "first.cu"), str(tmp_path / "calls.cpp"), "-o", exe, "-lpthread"], capture_output=True, text=True)
    if "cannot find -ltsan" in made.stderr or "libtsan" in made.stderr:
        pytest.skip("needs the thread sanitizer")
    assert made.returncode == 0, made.stderr
    ran = subprocess.run([exe], capture_output=True, text=True, env=dict(os.environ, TSAN_OPTIONS="halt_on_error=1"))
    if "unexpected memory mapping" in ran.stderr:
        pytest.skip("the thread sanitizer does not run here")
    assert ran.returncode == 0, (ran.returncode, ran.stderr[-3000:])
