"""Calls with one GPU current, then with another, and from threads at once, through the library on a HIP runtime of the test's own (no GPU): a launch is refused, as a runtime refuses it, where its
dynamic LDS is beyond what the current device has been told for that kernel."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2410_17043_amd import _lib

# What the library calls of the runtime on its way to a launch.  Nothing is executed; "device" memory is the host's.
RUNTIME = r"""
#include <hip/hip_runtime_api.h>
#include <chrono>
#include <cstdlib>
#include <map>
#include <mutex>
#include <thread>
#include <utility>
static thread_local int device = 0;
static thread_local hipError_t last = hipSuccess;
static thread_local dim3 grid, block;
static thread_local size_t lds;
static thread_local hipStream_t stream;
static std::mutex mutex;
static std::map<std::pair<int, const void*>, int> limits;
static int launches = 0, large = 0, raises = 0;
extern "C" {
int fake_launches() { return launches; }
int fake_large() { return large; }
int fake_raises() { return raises; }
void fake_device(int d) { device = d; }
hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { *p = std::malloc(n); return *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
hipError_t hipGetLastError() { const hipError_t e = last; last = hipSuccess; return e; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipFuncSetAttribute(const void* f, hipFuncAttribute, int bytes) {
    std::this_thread::sleep_for(std::chrono::milliseconds(2));
    std::lock_guard<std::mutex> lock(mutex);
    limits[{device, f}] = bytes;
    ++raises;
    return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t l, hipStream_t s) { grid = g; block = b; lds = l; stream = s; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* l, hipStream_t* s) { *g = grid; *b = block; *l = lds; *s = stream; return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3, dim3, void**, size_t l, hipStream_t) {
    std::lock_guard<std::mutex> lock(mutex);
    ++launches;
    if (l > 65536) ++large;
    auto it = limits.find({device, f});
    if (l > 65536 && (it == limits.end() || (size_t)it->second < l)) return last = hipErrorInvalidValue;
    return hipSuccess;
}
}
"""

# Runs in a process of its own, without torch (whose runtime is the real one)
CALLS = r"""
import ctypes as C, importlib.util, sys, threading
fake = C.CDLL(sys.argv[1], C.RTLD_GLOBAL)                       # in front of the real one
spec = importlib.util.spec_from_file_location("_lib", sys.argv[2])
B = importlib.util.module_from_spec(spec)
spec.loader.exec_module(B)
lib = C.CDLL(B.LIB_PATH)
for name, (res, args) in B.SIGNATURES.items():
    f = getattr(lib, name)
    f.restype, f.argtypes = res, args
some = C.c_void_p(1 << 32)                                      # an address that nothing follows
room = 1 << 40

def ffn(kind, R, H, F, act, n=1):
    table = {"bf16": B.moe_expert_w, "fp8": B.moe_expert_w8, "int8": B.moe_expert_wi8, "fp32": B.moe_expert_w}[kind]
    w = (table * n)()
    for e in w:
        for field, _ in table._fields_:
            setattr(e, field, some.value)
    if kind in ("bf16", "fp32"):
        return lib.moe_expert_ffn(some, R, some, some, n, w, n, H, F, act, 1 if kind == "bf16" else 0, some, some, room, None)
    return getattr(lib, "moe_expert_ffn_" + kind)(some, R, some, some, n, w, n, H, F, act, some, some, room, None)

def route(T, H, E, k, dtype):
    ctx, shape = C.c_void_p(), B.moe_shape(T, H, E, k, 1, dtype, 0, 0)
    assert lib.moe_ctx_create(C.byref(ctx), C.byref(shape)) == 0
    rc = lib.moe_route(ctx, some, some, None, some, some, None)
    if rc == 0 and H % 64 == 0:
        rule = B.moe_gate_rule()
        rule.n_groups = rule.top_groups = 1
        rule.scale = 1.0
        need = lib.moe_route_grouped_workspace_bytes(ctx, C.byref(rule))
        rc = lib.moe_route_grouped(ctx, some, some, C.byref(rule), None, some, some, some, max(need, 1 << 30), None)
    lib.moe_ctx_destroy(ctx)
    return rc

# every kind of FFN kernel and of gate that takes more than 64 KB
calls = [lambda a=a: ffn(*a) for kind in ("int8", "fp8", "bf16") for act in range(3) for a in
         [(kind, R, H, F, act, n) for R, H, F, n in ((5, 1024, 8192, 1), (20, 1024, 8192, 1), (60, 896, 8064, 1), (400, 1152, 640, 4), (403, 2048, 1408, 4), (700, 1152, 2304, 4),
                                                     (9000, 512, 256, 1), (9000, 1024, 1408, 1), (20571, 4096, 14336, 1), (1100, 128, 14336, 1))]]
calls += [lambda a=a: ffn(*a) for act in range(3) for a in (("fp32", 300, 256, 512, act, 2), ("fp32", 9000, 1024, 1408, act, 1))]
calls += [lambda a=a: route(*a) for T in (1, 40, 4096) for E in (8, 24, 64, 100, 256) for a in ((T, 2048, E, 4, 1), (T, 1024, E, 4, 0))]

def all_of(device):
    fake.fake_device(device)
    for i, c in enumerate(calls):
        rc = c()
        assert rc == 0, (device, i, rc, lib.moe_last_error())

if sys.argv[3] == "devices":
    all_of(0)
    large, raises = fake.fake_large(), fake.fake_raises()
    assert large > 40 and raises > 20, (large, raises)
    all_of(0)
    assert fake.fake_raises() == raises and fake.fake_large() == 2 * large   # told once
    all_of(1)
    assert fake.fake_raises() == 2 * raises and fake.fake_large() == 3 * large
    all_of(0)
    all_of(70)
    all_of(6)                                                   # (70 modulo 64)
else:
    failed = []
    def work(device):
        try:
            all_of(device)
        except BaseException as e:
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i % 2,)) for i in range(8)]
    for t in threads: t.start()
    for t in threads: t.join()
    assert not failed, failed[0]
print("fine", fake.fake_launches(), fake.fake_large(), fake.fake_raises())
"""


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    d = tmp_path_factory.mktemp("runtime")
    (d / "fake.cpp").write_text(RUNTIME)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-O1", "-shared", "-fPIC", "-pthread", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-o", str(d / "fake.so"),
                    str(d / "fake.cpp")], check=True)
    (d / "calls.py").write_text(CALLS)
    return d


@pytest.mark.parametrize("how", ["devices", "threads"])
def test_a_launch_is_never_beyond_its_devices_limit(runtime, how):
    p = subprocess.run([sys.executable, str(runtime / "calls.py"), str(runtime / "fake.so"), _lib.__file__, how], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.startswith("fine"), p.stdout + p.stderr
