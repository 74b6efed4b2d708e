"""A HIP runtime of nothing but bookkeeping, for tests of the library's host side without a GPU: allocations are numbers, launches names.

A child process loads it before the library (the calls of both runtimes' names then go to this one) and runs a test's code with `fake`, `L` (the library), `gtree`, `np`
and `shares` at hand; what the code prints is returned."""
import atexit
import functools
import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCE = r"""
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <map>
#include <string>
#include <vector>
typedef int E;                                    // hipError_t
struct Dim { uint32_t x, y, z; };
static std::map<uint64_t, size_t> live;
static std::map<const void *, std::string> names;
static std::vector<std::string> log_;
static uint64_t next_ = 1ull << 40;
static size_t now_, peak_, largest_;
static long fail_ = -1, tries_, bad_;
static int capturing_;
static struct { Dim g, b; size_t s; void *st; } call_;
extern "C" {
E hipMalloc(void **p, size_t n)
{
    if (capturing_) bad_++;
    if (tries_++ == fail_) return 2;
    *p = (void *)next_; live[next_] = n; next_ += (n + 4096) / 4096 * 4096;
    now_ += n; if (now_ > peak_) peak_ = now_; if (n > largest_) largest_ = n;
    return 0;
}
E hipFree(void *p)
{
    if (!p) return 0;
    if (capturing_) bad_++;
    auto it = live.find((uint64_t)p);
    if (it == live.end()) { bad_++; return 1; }
    now_ -= it->second; live.erase(it);
    return 0;
}
E hipMemset(void *, int, size_t) { return 0; }
E hipMemsetAsync(void *, int, size_t, void *) { if (capturing_) bad_++; return 0; }
E hipMemcpy(void *d, const void *, size_t n, int kind) { if (kind == 2) memset(d, 0, n); return 0; }
E hipGetDevice(int *d) { *d = 0; return 0; }
E hipDeviceGetAttribute(int *v, int, int) { *v = 256; return 0; }
E hipGetSymbolAddress(void **p, const void *) { *p = (void *)(1ull << 39); return 0; }
E hipStreamSynchronize(void *) { if (capturing_) bad_++; return 0; }
E hipDeviceSynchronize() { return 0; }
E hipStreamIsCapturing(void *, int *s) { *s = capturing_; return 0; }
E hipEventCreate(void **e) { *e = (void *)1; return 0; }
E hipEventDestroy(void *) { return 0; }
E hipEventRecord(void *, void *) { return 0; }
E hipEventElapsedTime(float *t, void *, void *) { *t = 0; return 0; }
E hipGetLastError() { return 0; }
E hipPeekAtLastError() { return 0; }
const char *hipGetErrorString(E) { return "fake"; }
E __hipPushCallConfiguration(Dim g, Dim b, size_t s, void *st) { call_ = { g, b, s, st }; return 0; }
E __hipPopCallConfiguration(Dim *g, Dim *b, size_t *s, void **st) { *g = call_.g; *b = call_.b; *s = call_.s; *st = call_.st; return 0; }
E hipLaunchKernel(const void *f, Dim g, Dim b, void **, size_t, void *)
{
    if (!g.x || !g.y || !g.z || (uint64_t)g.x * b.x >= 1ull << 32 || g.y > 65535 || g.z > 65535) bad_++;
    log_.push_back(names[f]);
    return 0;
}
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *f, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names[f] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
// the tests' side
void fake_fail(long at) { fail_ = at; tries_ = 0; }             // the at-th allocation from here on fails (-1: none)
long fake_tries() { return tries_; }
void fake_capture(int on) { capturing_ = on; }
size_t fake_now() { return now_; }
size_t fake_peak() { const size_t p = peak_; peak_ = now_; return p; }
size_t fake_largest() { const size_t p = largest_; largest_ = 0; return p; }
long fake_bad() { return bad_; }                                // frees of nothing, launches beyond the limits, waits and allocations under capture
int fake_live(uint64_t p) { return live.count(p) != 0; }
uint64_t fake_newest() { return live.empty() ? 0 : live.rbegin()->first; }
size_t fake_launches() { return log_.size(); }
const char *fake_launch(size_t i) { return log_[i].c_str(); }
}
"""
CHILD = r"""
import ctypes as C, sys
sys.path[:0] = [%(root)r, %(here)r]
fake = C.CDLL(%(so)r, mode=C.RTLD_GLOBAL)
for name in ("now", "peak", "largest", "newest", "launches"):
    getattr(fake, "fake_" + name).restype = C.c_size_t
fake.fake_fail.argtypes, fake.fake_tries.restype, fake.fake_bad.restype = [C.c_long], C.c_long, C.c_long
fake.fake_live.argtypes = [C.c_uint64]
fake.fake_launch.argtypes, fake.fake_launch.restype = [C.c_size_t], C.c_char_p
import numpy as np
from paper_2305_00645_amd import gtree
L = gtree.load()

def shares(n):
    s = gtree._Shares()
    for p in range(3):
        s.party[p].own = s.party[p].next = 1 << 38
    s.n = n
    return C.byref(s)

def context(flags=0, tau=16, stream=1):
    prm = gtree._Params()
    prm.tau, prm.K, prm.flags, prm.hip_stream = tau, 2, flags, stream
    h = C.c_void_p()
    assert L.gt_ctx_create(C.byref(h), C.byref(prm)) == 0
    return h

def counted(ctx):
    st = gtree._Stats()
    assert L.gt_stats_get(ctx, C.byref(st)) == 0
    return L.gt_op_counter(ctx), st.rounds, [int(st.wire_bytes[a][b]) for a in range(3) for b in range(3)]

def dense(ctx, din, dout):
    h = C.c_void_p()
    assert L.gt_dense_create(ctx, shares(din * dout), None, din, dout, C.byref(h)) == 0
    return h

def moe(ctx, d, ff, E, top, rows):
    h = C.c_void_p()
    assert L.gt_moe_create(ctx, shares(d * E), None, shares(E * d * ff), None, shares(E * d * ff), None, d, ff, E, top, rows, C.byref(h)) == 0
    return h
"""


@functools.lru_cache(None)
def _built():
    tmp = tempfile.mkdtemp()
    atexit.register(shutil.rmtree, tmp, True)
    src, so = os.path.join(tmp, "fake_hip.cpp"), os.path.join(tmp, "fake_hip.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", so, src], check=True)
    return so


def run(code):
    child = CHILD % dict(root=os.path.dirname(HERE), here=HERE, so=_built())
    r = subprocess.run([sys.executable, "-c", child + code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return r.stdout
