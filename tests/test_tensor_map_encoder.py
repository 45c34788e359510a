"""The tensor-map encoder is looked up once and by any number of host threads at a time (contexts on threads of
their own create caches and models): none may see it missing while another still looks.  On the CPU, with a driver
lookup that takes its time."""
import os
import subprocess

from paper_2607_18582_gb300 import build

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>
#include "tc_util.cuh"

static int lookups = 0;
extern "C" cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **fn, unsigned int, unsigned long long,
                                                        cudaDriverEntryPointQueryResult *q)
{
    ++lookups;
    std::this_thread::sleep_for(std::chrono::milliseconds(200));
    *fn = reinterpret_cast<void *>(&lookups);
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

int main()
{
    bool there[8] = {};
    std::vector<std::thread> threads;
    for (int i = 0; i < 8; ++i)
        threads.emplace_back([&, i] {
            std::this_thread::sleep_for(std::chrono::milliseconds(10 * i));
            there[i] = mure::tensor_map_encoder() != nullptr;
        });
    for (auto &t : threads) t.join();
    int n = 0;
    for (bool b : there) n += b;
    std::printf("%d %d\n", n, lookups);
    return 0;
}
"""


def test_threads_all_find_the_encoder(tmp_path):
    src, exe = tmp_path / "encoder.cu", tmp_path / "encoder"
    src.write_text(PROGRAM)
    nvcc = build._nvcc()
    r = subprocess.run([nvcc] + build.ARCH + ["-std=c++17", "-cudart", "shared", "-I", build.CSRC, "-I", build.INCLUDE,
                                              "-o", str(exe), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lib = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "lib64") if os.path.isabs(nvcc) else ""
    env = dict(os.environ, LD_LIBRARY_PATH=":".join(p for p in (lib, os.environ.get("LD_LIBRARY_PATH", "")) if p))
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60, env=env)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split() == ["8", "1"], r.stdout
