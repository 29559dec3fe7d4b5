"""The host side of the branching cache (csrc/xc_pool.cpp) on the CPU: compiled with the host compiler against
stand-ins for HIP's calls and for the kernels' launches, through the C ABI of include/xcache.h.

Device memory is a range of addresses that nobody reads.  Work is numbered as it is launched and counts as done once the
stream or an event behind it has been waited for.  Faults are asked for by number: the n-th allocation from now on, on
the device or by operator new, fails."""
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

from paper_2604_20289_amd import build, xcache

SHIM = r"""
#include "xc_pool.h"
#include "xcache.h"
#include <cstdlib>
#include <map>
#include <new>
#include <vector>
using namespace xc;
typedef unsigned long long u64;

// state of the stand-ins
static int device, capture, elsewhere, broken, device_fails = -1, new_fails = -1, launch_fails = -1;
static u64 most_bytes = ~0ull, next_address = 1ull << 44, launched, done;
struct Block { u64 bytes, used; };
static std::map<u64, Block>* blocks;
static std::map<void*, u64>* events;
static std::vector<int>* calls;
static int freed_in_use, freed_unknown, launched_on = -1;
static u64 live_bytes, peak_bytes;
static AttnArgs last_attention;

static hipStreamCaptureMode mode = hipStreamCaptureModeGlobal;
// while another stream is captured, this thread's mode decides whether allocations are let through or end that capture
static bool forbidden() {
  const bool f = elsewhere && mode != hipStreamCaptureModeRelaxed;
  if (f) ++broken;
  return f;
}

static bool counts_down(int& n) { return n >= 0 && n-- == 0; }
void* operator new(size_t n) {
  if (counts_down(new_fails)) throw std::bad_alloc();
  if (void* p = malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

static void use(const void* p) {
  const u64 at = (u64)p;
  auto it = blocks->upper_bound(at);
  if (it == blocks->begin()) return;
  --it;
  if (at < it->first + it->second.bytes) it->second.used = launched;
}
static hipError_t launch(int kind) {
  if (counts_down(launch_fails)) return hipErrorLaunchFailure;
  ++launched;
  launched_on = device;
  calls->push_back(kind);
  return hipSuccess;
}
static void finish(u64 to) { if (to > done) done = to; }

extern "C" {
hipError_t hipGetDevice(int* d) { return *d = device, hipSuccess; }
hipError_t hipSetDevice(int d) { return device = d, hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
hipError_t hipThreadExchangeStreamCaptureMode(hipStreamCaptureMode* m) { return std::swap(mode, *m), hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) {
  if (forbidden()) return hipErrorStreamCaptureUnsupported;
  if (counts_down(device_fails) || live_bytes + n > most_bytes) return hipErrorOutOfMemory;
  const int keep = new_fails;
  new_fails = -1;
  (*blocks)[next_address] = {n, 0};
  new_fails = keep;
  *p = (void*)next_address;
  next_address += (n + (1 << 20)) & ~0xffffull;
  live_bytes += n;
  if (live_bytes > peak_bytes) peak_bytes = live_bytes;
  return hipSuccess;
}
hipError_t hipFree(void* p) {
  if (forbidden()) return hipErrorStreamCaptureUnsupported;
  auto it = blocks->find((u64)p);
  if (it == blocks->end()) return ++freed_unknown, hipErrorInvalidValue;
  if (it->second.used > done) ++freed_in_use;
  live_bytes -= it->second.bytes;
  blocks->erase(it);
  return hipSuccess;
}
hipError_t hipHostMalloc(void** p, size_t n, unsigned) {
  if (forbidden()) return hipErrorStreamCaptureUnsupported;
  if (counts_down(device_fails)) return hipErrorOutOfMemory;
  return (*p = malloc(n)) ? hipSuccess : hipErrorOutOfMemory;
}
hipError_t hipHostFree(void* p) { return forbidden() ? hipErrorStreamCaptureUnsupported : (free(p), hipSuccess); }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return *e = (hipEvent_t)malloc(1), hipSuccess; }
hipError_t hipEventRecord(hipEvent_t e, hipStream_t) {
  const int keep = new_fails;
  new_fails = -1;
  (*events)[e] = launched;
  new_fails = keep;
  return hipSuccess;
}
hipError_t hipEventSynchronize(hipEvent_t e) { return finish((*events)[e]), hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t e) { return events->erase(e), free(e), hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return finish(launched), hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  return *s = capture ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone, hipSuccess;
}
hipError_t hipMemcpyAsync(void* d, const void*, size_t, hipMemcpyKind, hipStream_t) { return ++launched, use(d), hipSuccess; }

void fake_init() {
  blocks = new std::map<u64, Block>;
  events = new std::map<void*, u64>;
  calls = new std::vector<int>;
  calls->reserve(1 << 16);
}
void fake_reset() {
  device = capture = elsewhere = broken = freed_in_use = freed_unknown = 0;
  device_fails = new_fails = launch_fails = -1;
  most_bytes = ~0ull;
  peak_bytes = live_bytes;
  calls->clear();
}
void fake_set(int dev, int cap) { device = dev, capture = cap; }
void fake_elsewhere(int on) { elsewhere = on; }
void fake_faults(int dev, int host, int kernel) { device_fails = dev, new_fails = host, launch_fails = kernel; }
void fake_memory(u64 most) { most_bytes = most; }
u64 fake_info(int what) {
  const u64 v[] = {live_bytes, peak_bytes, (u64)freed_in_use, (u64)freed_unknown, blocks->size(), (u64)device,
                   (u64)calls->size(), (u64)last_attention.n_slots, (u64)(calls->empty() ? -1 : calls->back()),
                   (u64)(device_fails >= 0 || new_fails >= 0), (u64)launched_on, (u64)broken, (u64)mode};
  return v[what];
}
}

namespace xc {
hipError_t launch_page_copies(const PageCopy*, int, const PageBuf&, int, int, long long, hipStream_t) { return launch(0); }
hipError_t launch_import(const ImportArgs&, const HandleWindow&, int, int, int, int, const PageBuf&, long long, hipStream_t) {
  return launch(1);
}
hipError_t launch_batch_rows(const int* tables, const BatchSeq*, int, int, int, int*, OwnSlots*, hipStream_t) {
  const hipError_t e = launch(2);
  use(tables);
  return e;
}
hipError_t launch_norm_rope(int, const NormRopeArgs& a, hipStream_t) {
  const hipError_t e = launch(3);
  use(a.place);
  return e;
}
hipError_t launch_branch_attention(int, const AttnArgs& a, hipStream_t) {
  const hipError_t e = launch(4);
  last_attention = a;
  use(a.tables);
  if (a.n_slots) use(a.pieces);
  return e;
}
HandleWindow handle_window(const xc_handle*) { return {}; }
}  // namespace xc
extern "C" const char* xc_status_string(xc_status) { return "refused"; }
"""
INFO = ("live_bytes", "peak_bytes", "freed_in_use", "freed_unknown", "blocks", "device", "launches", "n_slots", "last_launch",
        "fault_ahead", "launched_on", "broken_captures", "mode")


@functools.lru_cache(None)
def lib():
    d = tempfile.mkdtemp(prefix="xc_pool_")
    src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    # (what the headers give to kernels alone is no concern of the host compiler's; the stand-ins are bound within)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-D_GLIBCXX_ASSERTIONS", "-D__HIP_PLATFORM_AMD__", "-D__bf16=short",
                    "-w", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-isystem", "/opt/rocm/include", "-I", build.INCLUDE, "-I",
                    build.CSRC, src, os.path.join(build.CSRC, "xc_pool.cpp"), "-o", so], check=True)
    out = ctypes.CDLL(so)
    for name in xcache.EXPORTED:
        if name.startswith(("xc_pool", "xc_seq", "xc_batch", "xc_qk_norm_rope", "xc_branch")):
            mine, theirs = getattr(out, name), getattr(xcache.load_library(), name)
            mine.restype, mine.argtypes = theirs.restype, theirs.argtypes
    out.fake_info.restype = ctypes.c_ulonglong
    out.fake_memory.argtypes = [ctypes.c_ulonglong]
    out.fake_init()
    return out


def info():
    return {name: lib().fake_info(i) for i, name in enumerate(INFO)}


def ints(*x):
    return (ctypes.c_int32 * len(x))(*x)


KEYS, VALUES, ROWS = 1 << 40, 1 << 41, 1 << 42  # addresses of the caller's buffers


class HostPool:
    """A pool of the C ABI over buffers that are addresses alone."""

    def __init__(self, n_blocks=1, q_heads=1, kv_heads=1, head_dim=64, dtype=xcache.XC_BF16, page_tokens=16, n_pages=64,
                 max_seqs=64):
        lib().fake_reset()
        self.c = xcache.PoolConfigC(n_blocks, q_heads, kv_heads, head_dim, dtype, page_tokens, n_pages, max_seqs)
        p = ctypes.c_void_p()
        assert lib().xc_pool_init(ctypes.byref(self.c), KEYS, VALUES, None, ctypes.byref(p)) == xcache.XC_OK
        self.p = p.value

    def new(self, tokens=0):
        s = ctypes.c_int32()
        assert lib().xc_seq_new(self.p, ctypes.byref(s)) == xcache.XC_OK
        if tokens:
            assert lib().xc_seq_extend(self.p, 1, ints(s.value), ints(tokens)) == xcache.XC_OK
        return s.value

    def fork(self, src, n):
        out = ints(*[0] * n)
        assert lib().xc_seq_fork(self.p, src, n, out) == xcache.XC_OK
        return list(out)

    def batch(self):
        b = ctypes.c_void_p()
        assert lib().xc_batch_init(self.p, ctypes.byref(b)) == xcache.XC_OK
        return b.value

    def close(self):
        lib().fake_faults(-1, -1, -1)
        assert lib().xc_pool_destroy(self.p) == xcache.XC_OK


def set_batch(b, seqs, new):
    return lib().xc_batch_set(b, len(seqs), ints(*seqs), ints(*new))


def attention(b, width=64, q=ROWS, out=ROWS + (1 << 38), block=0):
    return lib().xc_branch_attention(b, block, q, width, 0.0, out, width)


class Tensor:
    """What the binding asks of a page buffer."""

    class Device:
        type = "cuda"

        def __init__(self, index):
            self.index = index

        def __eq__(self, other):
            return self.index == other.index

    def __init__(self, at, shape, device=0):
        self.at, self.shape, self.dtype, self.device = at, shape, "torch.bfloat16", Tensor.Device(device)

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def get_device(self):
        return self.device.index
