"""Page tables of the branching cache, plainly: dictionaries and sets, one
token at a time, and the host code (csrc/xc_pages.h) compiled with the host
compiler and called through ctypes."""
import ctypes
import functools
import os
import subprocess
import tempfile

from paper_2604_20289_amd import build

SHIM = r"""
#include "xc_pages.h"
using namespace xc;
static std::vector<PageCopy> copies;
extern "C" {
void* book_new(int n_pages, int shift, int max_seqs) { return new PageBook(n_pages, shift, max_seqs); }
void book_delete(void* b) { delete (PageBook*)b; }
int book_create(void* b, int* out) { return (int)((PageBook*)b)->create(out); }
int book_fork(void* b, int src, int n, int* out) { return (int)((PageBook*)b)->fork(src, n, out); }
int book_extend(void* b, int n, const int* s, const int* t) { return (int)((PageBook*)b)->extend(n, s, t, &copies); }
int book_trim(void* b, int s, int front, int back) { return (int)((PageBook*)b)->trim(s, front, back); }
int book_free(void* b, int n, const int* s) { return (int)((PageBook*)b)->free(n, s); }
void book_compact(void* b) { ((PageBook*)b)->compact(&copies); }
int n_copies() { return (int)copies.size(); }
void get_copies(int* out) { for (auto& c : copies) *out++ = c.src, *out++ = c.dst, *out++ = c.rows; }
int book_refs(void* b, int p) { return ((PageBook*)b)->refs(p); }
int book_live(void* b) { return ((PageBook*)b)->live_pages(); }
int book_seqs(void* b) { return ((PageBook*)b)->live_seqs(); }
int book_get(void* b, int s, int* first, int* tokens, int* pages) {
  if (!((PageBook*)b)->valid(s)) return -1;
  const PageSeq& q = ((PageBook*)b)->seq(s);
  *first = q.first, *tokens = q.tokens;
  for (int p : q.pages) *pages++ = p;
  return (int)q.pages.size();
}
unsigned long long book_version(void* b, int s) { return ((PageBook*)b)->seq(s).version; }
}
"""
OK, INVALID, FULL = range(3)


@functools.lru_cache(None)
def lib():
    d = tempfile.mkdtemp(prefix="xc_pages_")
    src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-D_GLIBCXX_ASSERTIONS", "-Wall", "-Werror", "-shared", "-fPIC",
                    "-I", build.CSRC, src, "-o", so], check=True)
    out = ctypes.CDLL(so)
    out.book_new.restype = ctypes.c_void_p
    out.book_version.restype = ctypes.c_ulonglong
    for name in ("book_delete", "book_create", "book_fork", "book_extend", "book_trim", "book_free", "book_compact",
                 "book_refs", "book_live", "book_seqs", "book_get"):
        getattr(out, name).argtypes = None
    return out


def ints(x):
    return (ctypes.c_int * len(x))(*x)


class Book:
    """The host code."""

    def __init__(self, n_pages, shift, max_seqs):
        self.n_pages, self.max_seqs = n_pages, max_seqs
        self.b = ctypes.c_void_p(lib().book_new(n_pages, shift, max_seqs))

    def __del__(self):
        lib().book_delete(self.b)

    def create(self):
        out = ctypes.c_int(-1)
        return lib().book_create(self.b, ctypes.byref(out)), out.value

    def fork(self, src, n):
        out = (ctypes.c_int * max(n, 0))()
        return lib().book_fork(self.b, src, n, out), list(out)

    def extend(self, seqs, tokens):
        s = lib().book_extend(self.b, len(seqs), ints(seqs), ints(tokens))
        return s, self._copies() if s == OK else None

    def trim(self, seq, front, back):
        return lib().book_trim(self.b, seq, front, back)

    def free(self, seqs):
        return lib().book_free(self.b, len(seqs), ints(seqs))

    def compact(self):
        lib().book_compact(self.b)
        return self._copies()

    def _copies(self):
        n = lib().n_copies()
        out = (ctypes.c_int * (3 * n))()
        lib().get_copies(out)
        return [tuple(out[3 * i:3 * i + 3]) for i in range(n)]

    def get(self, seq):
        first, tokens = ctypes.c_int(), ctypes.c_int()
        pages = (ctypes.c_int * self.n_pages)()
        n = lib().book_get(self.b, seq, ctypes.byref(first), ctypes.byref(tokens), pages)
        return None if n < 0 else (first.value, tokens.value, list(pages[:n]))

    def refs(self):
        return [lib().book_refs(self.b, p) for p in range(self.n_pages)]

    def version(self, seq):
        return lib().book_version(self.b, seq)

    def state(self):
        return ([self.get(s) for s in range(self.max_seqs)], self.refs(), lib().book_live(self.b),
                lib().book_seqs(self.b))
