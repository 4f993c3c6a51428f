"""What the library's entry points launch, without a GPU: a stand-in for the HIP runtime takes the launches of a child process down and runs none."""
import ctypes
import functools
import json
import os
import subprocess
import sys
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = os.environ.get("ROCM_PATH", "/opt/rocm") + "/include"

SOURCE = r"""
#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime_api.h>
#include <map>
#include <string>
#include <string.h>
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
static void (*take)(const char*, long long*) = nullptr;
static dim3 g_grid, g_block;
static size_t g_lds;
static hipStream_t g_stream;
extern "C" {
void set_take(void (*f)(const char*, long long*)) { take = f; }
static void tell(const void* f, long long kind, long long a, long long b, long long c, long long d, long long e, long long g, long long h) {
    long long v[8] = {kind, a, b, c, d, e, g, h};
    if (take) take(names()[f].c_str(), v);
}
void** __hipRegisterFatBinary(const void*) { static void* p; return &p; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, dim3*, dim3*, int*) { names()[host] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t s) { g_grid = grid; g_block = block; g_lds = lds; g_stream = s; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) { *grid = g_grid; *block = g_block; *lds = g_lds; *s = g_stream; return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3 g, dim3 b, void**, size_t lds, hipStream_t) { tell(f, 0, g.x, g.y, g.z, b.x, b.y, b.z, (long long)lds); return hipSuccess; }
hipError_t hipFuncSetAttribute(const void* f, hipFuncAttribute a, int value) {
    if (a == hipFuncAttributeMaxDynamicSharedMemorySize) tell(f, 1, value, 0, 0, 0, 0, 0, 0);
    return hipSuccess;
}
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t* p, int) { memset(p, 0, sizeof *p); strcpy(p->gcnArchName, "gfx950"); return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "none"; }
hipError_t hipGetSymbolAddress(void** p, const void*) { *p = nullptr; return hipErrorInvalidValue; }
}
"""


def child(runtime, library, calls):
    """in the child: [[status, [limits of LDS set: (kernel, bytes)], [launches: (kernel, grid, block, bytes of LDS)]] per call]"""
    shim = ctypes.CDLL(runtime, mode=ctypes.RTLD_GLOBAL)                 # before the library, whose names are looked up there first
    L = ctypes.CDLL(library)
    out, limits, launches = [], [], []

    @ctypes.CFUNCTYPE(None, ctypes.c_char_p, ctypes.POINTER(ctypes.c_longlong))
    def take(name, v):
        name = name.decode()
        if v[0]:
            limits.append((name, v[1]))
        else:
            launches.append((name, v[1:4], v[4:7], v[7]))
    shim.set_take(take)
    kinds = {"i": ctypes.c_int, "l": ctypes.c_longlong, "p": ctypes.c_void_p}
    for entry, signature, args in calls:
        del limits[:], launches[:]
        status = getattr(L, entry)(*[kinds[k](a) for k, a in zip(signature, args)])
        out.append([status, list(limits), list(launches)])
    return out


@functools.lru_cache(maxsize=None)
def _runtime():
    d = tempfile.mkdtemp()
    src, so = os.path.join(d, "launches.cpp"), os.path.join(d, "launches.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-I" + ROCM_INCLUDE, src, "-o", so], check=True)
    return so


def launches(calls):
    """calls: [(entry point, "iilp..." its arguments, them)] -> as child()"""
    from paper_2306_07629_amd import build
    if build.is_stale():
        build.build()
    run = subprocess.run([sys.executable, os.path.abspath(__file__), _runtime(), build.LIB], input=json.dumps(calls), capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
    return json.loads(run.stdout)


def is_possible(launch, limit=65536):
    """whether a launch stays within what the hardware and the runtime count: 1024 threads to a workgroup, 2^32 along a grid's axis, 65535 workgroups along y and z,
    the dynamic LDS that was asked for (64 KB without asking)"""
    _, grid, block, lds = launch
    threads = block[0] * block[1] * block[2]
    return (0 < threads <= 1024 and all(g > 0 and g * b < 1 << 32 for g, b in zip(grid, block)) and max(grid[1:]) <= 65535
            and 0 <= lds <= max(65536, limit) and lds <= 160 * 1024)


if __name__ == "__main__":
    print(json.dumps(child(sys.argv[1], sys.argv[2], json.load(sys.stdin))))
