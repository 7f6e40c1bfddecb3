"""The library's C interface over a device that is not there: argument checks, plans, workspace bookkeeping and locks
are the library's own, a launch is a line in a log.  "Device" addresses are host memory."""
import ctypes
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2512_12949_amd import binding as ff

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_12949_amd", "csrc")
STUB = r"""
#include <chrono>
#include <condition_variable>
#include <cstring>
#include <mutex>
#include <string>
#include "ffuse_launch.h"
namespace {
std::mutex mu;
std::condition_variable cv;
std::string lines, hold;
int count, capturing;
bool held;
hipError_t launched(const char* name) {
    std::unique_lock<std::mutex> lock(mu);
    lines += std::string(name) + " ";
    const int mine = ++count;
    cv.notify_all();
    if (hold == name && !held) {      // the first of its kind takes its time: until another launch, or half a second
        held = true;
        cv.wait_for(lock, std::chrono::milliseconds(500), [&] { return count > mine; });
        lines += "held ";
    }
    return hipSuccess;
}
}
extern "C" {
void stub_reset(const char* h, int c) { std::lock_guard<std::mutex> lock(mu); hold = h; lines.clear(); count = 0; held = false; capturing = c; }
int stub_held() { std::lock_guard<std::mutex> lock(mu); return held; }
int stub_log(char* out, int n) { std::lock_guard<std::mutex> lock(mu); std::strncpy(out, lines.c_str(), n - 1); return (int)lines.size(); }

hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) {
    std::memset(p, 0, sizeof(*p));
    std::strcpy(p->gcnArchName, "gfx950");
    p->multiProcessorCount = 256;
    return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { std::memcpy(d, s, n); return hipSuccess; }
hipError_t hipEventCreate(hipEvent_t*) { return hipErrorNotSupported; }
hipError_t hipEventDestroy(hipEvent_t) { return hipErrorNotSupported; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipErrorNotSupported; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipErrorNotSupported; }
hipError_t hipEventElapsedTime(float*, hipEvent_t, hipEvent_t) { return hipErrorNotSupported; }
hipError_t hipGetSymbolAddress(void**, const void*) { return hipErrorNotSupported; }
void** __hipRegisterFatBinary(const void*) { return nullptr; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void**) {}
}
namespace ffuse {
hipError_t launch_zero(void* p, size_t n, hipStream_t) { std::memset(p, 0, n); return launched("zero"); }
hipError_t launch_finalize(int, float*, void*, int64_t, hipStream_t) { return launched("finalize"); }
hipError_t launch_fused_f32(const FusedArgs&, float*, hipStream_t) { return launched("f32"); }
hipError_t launch_fused_rows(int, const RowsArgs&, int, int, int, hipStream_t) { return launched("rows"); }
hipError_t launch_fused_direct(int, const DirectArgs&, int, int, int, hipStream_t) { return launched("direct"); }
hipError_t launch_fused_reduce(int, const FusedArgs&, int, int, hipStream_t) { return launched("reduce"); }
hipError_t launch_fused_stream(int, const TwoPhaseArgs&, int, int, hipStream_t) { return launched("stream"); }
hipError_t launch_gemm_act_f32(const GemmArgs&, hipStream_t) { return launched("gemm"); }
hipError_t launch_fused_exchange(int, const ExchangeArgs&, int, hipStream_t) { return launched("exchange"); }
hipError_t launch_finalize_planes(int, const float*, void*, int64_t, int, hipStream_t) { return launched("planes"); }
hipError_t launch_fused_two_phase(int, const TwoPhaseArgs&, int, int, int, int, hipStream_t) { return launched("two_phase"); }
hipError_t launch_grouped_forward(int, const GroupedArgs& a, int, hipStream_t) {
    std::memset(a.C, 0x3f, (size_t)a.R * a.N * 2);
    return launched("grouped");
}
hipError_t launch_grouped_input(int, const GroupedArgs&, int, hipStream_t) { return launched("input"); }
hipError_t launch_grouped_weights(int, const GroupedArgs&, int, hipStream_t) { return launched("weights"); }
hipError_t launch_fp8_product(int, const Fp8Args&, int, hipStream_t) { return launched("fp8"); }
hipError_t launch_fp8_quantize(int, const void*, int64_t, int64_t, int, bool, void*, float*, hipStream_t) { return launched("quantize"); }
}
"""
SOURCES = ("ffuse_api", "ffuse_grouped_api", "ffuse_plan")


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def build(d):
    """The stubbed library, built in directory d."""
    if shutil.which("hipcc") is None or shutil.which("g++") is None:
        pytest.skip("no compiler")
    (d / "stub.cpp").write_text(STUB)
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("hipcc")))), "include")
    jobs = [["hipcc", "-x", "hip", "-O1", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-w", "-c", os.path.join(CSRC, s + ".cpp"), "-o", str(d / (s + ".o"))]
            for s in SOURCES]
    jobs.append(["g++", "-O1", "-std=c++17", "-fPIC", "-w", "-D__HIP_PLATFORM_AMD__", "-I", include, "-I", CSRC, "-c", str(d / "stub.cpp"), "-o", str(d / "stub.o")])
    with ThreadPoolExecutor(4) as pool:
        list(pool.map(_run, jobs))
    so = str(d / "stubbed.so")
    _run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", so, *(str(d / (s + ".o")) for s in SOURCES), str(d / "stub.o"), "-lpthread"])
    L = ctypes.CDLL(so, mode=os.RTLD_NOW | os.RTLD_LOCAL)
    real = ff.lib()
    for name in ff.EXPORTS:
        if hasattr(L, name):
            getattr(L, name).restype, getattr(L, name).argtypes = getattr(real, name).restype, getattr(real, name).argtypes
    L.stub_reset.argtypes = [ctypes.c_char_p, ctypes.c_int]
    L.stub_log.argtypes = [ctypes.c_char_p, ctypes.c_int]
    return L


def log(L):
    out = ctypes.create_string_buffer(1 << 16)
    L.stub_log(out, len(out))
    return out.value.decode().split()
