"""The persistent kernels of the products by expert and of the 8-bit products: no more workgroups than the CUs hold at a
time, for any problem, and a launch that the device takes.  The launches' host code over a runtime that only notes them."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_12949_amd", "csrc")
STUB = r"""
#include <cstdio>
#include <map>
#include <string>
#include "ffuse_launch.h"
%s
namespace {
std::map<const void*, std::string> names;
dim3 grid, block;
size_t lds;
std::string last;
}
extern "C" {
void** __hipRegisterFatBinary(const void*) { return nullptr; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names[f] = name; }
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t l, hipStream_t) { grid = g; block = b; lds = l; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* l, hipStream_t* s) { *g = grid; *b = block; *l = lds; *s = nullptr; return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3 g, dim3 b, void**, size_t l, hipStream_t) {
    last = names[f] + " " + std::to_string(g.x) + " " + std::to_string(b.x) + " " + std::to_string(l);
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
// kind: 0 forward, 1 gated, 2 the gradient of the input, 3 of the weights, 4 / 5 in 8 bits with b_block 1 / 128
const char* launched(int kind, int R, int E, int K, int N) {
    static char any[16];
    last.clear();
    const ffuse::GroupedArgs g{any, any, kind == 1 ? any : nullptr, reinterpret_cast<int32_t*>(any), any, R, E, K, N, 0};
    const ffuse::Fp8Args f{any, nullptr, any, nullptr, E > 0 ? reinterpret_cast<int32_t*>(any) : nullptr, any, R, E > 0 ? E : 1, K, N, kind == 4 ? 1 : 128};
    if (kind < 2) ffuse::launch_grouped_forward(0, g, 256, nullptr);
    else if (kind == 2) ffuse::launch_grouped_input(0, g, 256, nullptr);
    else if (kind == 3) ffuse::launch_grouped_weights(0, g, 256, nullptr);
    else ffuse::launch_fp8_product(0, f, 256, nullptr);
    return last.c_str();
}
}
"""


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return r.stdout


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("hipcc") is None or shutil.which("g++") is None:
        pytest.skip("no compiler")
    d = tmp_path_factory.mktemp("launches")
    objects, symbols = [], []
    for s in ("ffuse_grouped", "ffuse_fp8"):
        objects.append(str(d / (s + ".o")))
        _run(["hipcc", "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-w", "-c", os.path.join(CSRC, s + ".hip"), "-o", objects[-1]])
        symbols += re.findall(r"__hip_fatbin\w*", _run(["nm", "-u", objects[-1]]))
    (d / "stub.cpp").write_text(STUB % "\n".join(f'extern "C" {{ char {s}[16]; }}' for s in symbols))
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("hipcc")))), "include")
    _run(["g++", "-shared", "-Wl,-Bsymbolic", "-O1", "-std=c++17", "-fPIC", "-w", "-D__HIP_PLATFORM_AMD__", "-I", include, "-I", CSRC, str(d / "stub.cpp"), *objects,
          "-o", str(d / "launches.so")])
    L = ctypes.CDLL(str(d / "launches.so"), mode=os.RTLD_NOW | os.RTLD_LOCAL)
    L.launched.restype = ctypes.c_char_p
    return L


_KERNELS = {}


def _kernel(name):
    """(family, LDS bytes of its own, threads) of a kernel, from its template's arguments in its mangled name."""
    if name not in _KERNELS:
        family = re.match(r"_ZN5ffuse\d+(\w+?)_kernelI", name).group(1)
        most, waves = 0, 8
        for gemm, flags, numbers in re.findall(r"(PairGemm|Fp8Gemm)I\w+?((?:Lb[01]E)*)((?:Li\d+E){5})", name):
            gated = gemm == "PairGemm" and flags.endswith("Lb1E")
            bm, bn, wm, wn, ns = (int(n) for n in re.findall(r"\d+", numbers))
            waves, wide = wm * wn, bn // wn
            stage = (bm + (2 if gated else 1) * bn) * 128 + (((bm + 63) // 64 + (bn + 63) // 64) * 256 if gemm == "Fp8Gemm" else 0)
            out = 32 if wide == 64 and ns * stage + waves * 2048 > 152 * 1024 else wide
            most = max(most, ns * stage + waves * 32 * out)
        assert most or family == "fp8_stream", name
        _KERNELS[name] = family, most, 64 * waves
    return _KERNELS[name]


def _launch(lib, *problem):
    name, grid, block, table = lib.launched(*problem).decode().split()
    return (*_kernel(name), int(grid), int(block), int(table))


@pytest.mark.parametrize("kind", (0, 1, 2, 4, 5))
def test_as_many_workgroups_as_the_device_holds(lib, kind):
    rng, seen = random.Random(kind), set()
    for i in range(3000):
        E = rng.choice((1, rng.randint(2, 64), rng.randint(65, 512), rng.randint(513, 1024), 1024))
        R = int(2 ** rng.uniform(0, 16))
        K, N = (16 * int(2 ** rng.uniform(0, 8)) for _ in range(2))
        family, lds, threads, grid, block, table = _launch(lib, kind, R, E, K, N)
        if family == "fp8_stream":      # (not a persistent one)
            continue
        assert block == threads and table == 8 * E and grid % 8 == 0
        held = 160 * 1024 // (lds + table)
        assert held >= 1 and grid <= 256 * held, (R, E, K, N, lds, table, grid)
        seen.add(lds)
    assert len(seen) >= 4
