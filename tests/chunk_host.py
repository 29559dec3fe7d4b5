"""The host side of chunks under a mask (csrc/xc_chunk.cpp) on the CPU, beside that of the branching cache: as
tests/pool_host.py has it, with stand-ins for two more launches."""
import ctypes
import functools
import os
import subprocess
import tempfile

import pool_host as host
from paper_2604_20289_amd import build, xcache

SHIM = host.SHIM + r"""
#include "xc_chunk.h"
namespace xc {
hipError_t launch_weights(int, const WeightArgs& a, hipStream_t) {
  const hipError_t e = launch(5);
  use(a.tables);
  if (a.n_units) use(a.parts);
  return e;
}
hipError_t launch_evict(const EvictArgs& a, const Little*, const PageBuf&, int, int, long long, int, int, hipStream_t) {
  const hipError_t e = launch(6);
  use(a.seqs);
  use(a.src);
  return e;
}
}  // namespace xc
"""


@functools.lru_cache(None)
def lib():
    d = tempfile.mkdtemp(prefix="xc_chunk_")
    src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-D_GLIBCXX_ASSERTIONS", "-D__HIP_PLATFORM_AMD__", "-D__bf16=short",
                    "-w", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-isystem", "/opt/rocm/include", "-I", build.INCLUDE, "-I",
                    build.CSRC, src, *(os.path.join(build.CSRC, f) for f in ("xc_pool.cpp", "xc_chunk.cpp")), "-o", so],
                   check=True)
    out = ctypes.CDLL(so)
    for name in xcache.EXPORTED:
        if name.startswith(("xc_pool", "xc_seq", "xc_batch", "xc_qk_norm_rope", "xc_branch", "xc_chunk")):
            mine, theirs = getattr(out, name), getattr(xcache.load_library(), name)
            mine.restype, mine.argtypes = theirs.restype, theirs.argtypes
    out.fake_info.restype = ctypes.c_ulonglong
    out.fake_memory.argtypes = [ctypes.c_ulonglong]
    out.fake_init()
    return out


def info():
    return {name: lib().fake_info(i) for i, name in enumerate(host.INFO)}


KEYS, VALUES, ROWS, WEIGHTS, KEPT, LSE = (1 << 40, 1 << 41, 1 << 42, 1 << 43, (1 << 43) + (1 << 42), (1 << 43) + (1 << 41))


class Pool:
    """A pool and a batch of the C ABI over buffers that are addresses alone."""

    def __init__(self, **config):
        lib().fake_reset()
        c = dict(n_blocks=1, q_heads=1, kv_heads=1, head_dim=64, dtype=xcache.XC_BF16, page_tokens=16, n_pages=64, max_seqs=64)
        c.update(config)
        self.c = xcache.PoolConfigC(**c)
        p, b = ctypes.c_void_p(), ctypes.c_void_p()
        assert lib().xc_pool_init(ctypes.byref(self.c), KEYS, VALUES, None, ctypes.byref(p)) == xcache.XC_OK
        assert lib().xc_batch_init(p.value, ctypes.byref(b)) == xcache.XC_OK
        self.p, self.b, self.width = p.value, b.value, c["q_heads"] * c["head_dim"]

    def new(self, tokens=0):
        s = ctypes.c_int32()
        assert lib().xc_seq_new(self.p, ctypes.byref(s)) == xcache.XC_OK
        if tokens:
            assert lib().xc_seq_extend(self.p, 1, host.ints(s.value), host.ints(tokens)) == xcache.XC_OK
        return s.value

    def fork(self, src, n):
        out = host.ints(*[0] * n)
        assert lib().xc_seq_fork(self.p, src, n, out) == xcache.XC_OK
        return list(out)

    def table(self, s, cap=4096):
        first, tokens, count, pages = host.ints(0), host.ints(0), (ctypes.c_size_t * 1)(), host.ints(*[0] * cap)
        if lib().xc_seq_pages(self.p, s, first, tokens, pages, cap, count) != xcache.XC_OK:
            return None
        return first[0], tokens[0], list(pages[:count[0]])

    def tables(self):
        live = [ctypes.c_int32() for _ in range(3)]
        assert lib().xc_pool_info(self.p, *map(ctypes.byref, live)) == xcache.XC_OK
        return [self.table(s) for s in range(self.c.max_seqs)], [x.value for x in live]

    def set(self, seqs, new, group=1, window=0, sinks=0):
        m = xcache.ChunkMaskC(group, window, sinks)
        return lib().xc_chunk_set(self.b, len(seqs), host.ints(*seqs), host.ints(*new), ctypes.byref(m))

    def attention(self, q=ROWS, out=ROWS + (1 << 38), lse=LSE, ld=None, out_ld=None, scale=0.0, block=0):
        return lib().xc_chunk_attention(self.b, block, q, self.width if ld is None else ld, scale, out,
                                        self.width if out_ld is None else out_ld, lse)

    def weights(self, q=ROWS, lse=LSE, w=WEIGHTS, ld=1 << 20, q_ld=None, decay=1.0, scale=0.0, block=0):
        return lib().xc_chunk_weights(self.b, block, q, self.width if q_ld is None else q_ld, scale, lse, decay, w, ld)

    def evict(self, seqs, keep, sinks=0, recent=0, w=WEIGHTS, ld=1 << 20, kept=KEPT, kept_ld=1 << 20):
        return lib().xc_chunk_evict(self.b, len(seqs), host.ints(*seqs), host.ints(*keep), sinks, recent, w, ld, kept, kept_ld)

    def close(self):
        lib().fake_faults(-1, -1, -1)
        assert lib().xc_batch_destroy(self.b) == xcache.XC_OK
        assert lib().xc_pool_destroy(self.p) == xcache.XC_OK
        assert info()["blocks"] == 0 and info()["freed_unknown"] == 0 and info()["freed_in_use"] == 0
