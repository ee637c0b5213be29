"""What the library remembers per device, compiled from its source against stand-ins for the CUDA calls."""
import ctypes
import os
import subprocess

from rows_on_cpu import CSRC, _definition

FAKES = """
#include <atomic>
#include <algorithm>
#include <cstddef>
enum cudaError_t { cudaSuccess, cudaErrorUnknown };
enum { cudaFuncAttributeMaxDynamicSharedMemorySize };
struct cudaLaunchConfig_t {};
static int calls, answer;
static bool fails;
static cudaError_t cudaFuncSetAttribute(const void *, int, int) { ++calls; return fails ? cudaErrorUnknown : cudaSuccess; }
static cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *, const cudaLaunchConfig_t *) { ++calls; *n = answer; return fails ? cudaErrorUnknown : cudaSuccess; }
"""


def compiled(tmp_path, code):
    src, lib = tmp_path / "x.cpp", tmp_path / "x.so"
    src.write_text(FAKES + code)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-o", str(lib), str(src)], check=True)
    return ctypes.CDLL(str(lib))


def test_the_shared_memory_limit_is_raised_on_every_device(tmp_path):
    rows = open(os.path.join(CSRC, "tli_rows.cu")).read()
    lib = compiled(tmp_path, _definition(rows, "struct SmemAllowed") + """
extern "C" int ask(int device, int fail) {                                   // calls that reached CUDA, -1 for an error
    static SmemAllowed allowed;
    calls = 0; fails = fail;
    return allowed.set(nullptr, 100, device) == cudaSuccess ? calls : -1;
}""")
    assert [lib.ask(d, 0) for d in (64, 0, 0, 63, 63, 64, 1)] == [1, 1, 0, 1, 0, 1, 1]
    assert [lib.ask(2, f) for f in (1, 0, 0)] == [-1, 1, 0]


def test_resident_clusters_are_those_of_the_device(tmp_path):
    embed = open(os.path.join(CSRC, "tli_embed.cu")).read()
    lib = compiled(tmp_path, _definition(embed, "struct ClustersResident") + """
extern "C" int ask(int device, int clusters, int fail) {                     // (calls that reached CUDA, -1 for an error) * 1000 + clusters
    static ClustersResident resident;
    cudaLaunchConfig_t cfg;
    calls = 0; answer = clusters; fails = fail;
    int n = 0;
    return resident.get(nullptr, &cfg, device, n) == cudaSuccess ? calls * 1000 + n : -1;
}""")
    assert [lib.ask(d, c, 0) for d, c in ((0, 14), (1, 8), (0, 9), (1, 9), (64, 5), (0, 9), (63, 1))] == [1014, 1008, 14, 8, 1005, 14, 1002]
    assert [lib.ask(2, 7, f) for f in (1, 0, 0)] == [-1, 1007, 7]
