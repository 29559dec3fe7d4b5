"""Chunks under a mask at the largest sizes that include/xcache.h allows, on the CPU: what no test on a GPU has memory for."""
import ctypes
import shutil
import subprocess

import pytest

import chunk_host as chunk
import pool_host as host
from paper_2604_20289_amd import build
from paper_2604_20289_amd.xcache import XC_BF16, XC_ERR_OOM, XC_ERR_UNSUPPORTED, XC_F32, XC_OK

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")

TILES = r"""
#include "xc_chunk_plan.h"
#include <cstdio>
using namespace xc;

// a tile lies in rows `all` iff each of its 32 query rows is one of theirs
static bool truth(const RowRange& all, int r0, long long n, int group, long long tile) {
  if ((tile + 1) * 32 > n) return false;
  for (long long i = tile * 32; i < tile * 32 + 32; ++i)
    if (r0 + i / group < all.begin || r0 + i / group >= all.end) return false;
  return true;
}
int main() {
  const int most = 1 << 24;
  for (int group : {1, 3, 29, 64, 100, 128, 255, 256})
    for (int r0 : {0, 1, 777, (1 << 23) - 100, most - 4096 / group - 5})
      for (int rows : {1, 2, 31, 4096 / group + 1})
        for (int begin : {0, r0 - 1, r0, r0 + 1, r0 + rows / 2, r0 + rows, r0 + rows + 1, 1 << 23, (1 << 23) + 1, most - 1, most})
          for (int end : {0, r0, r0 + 1, r0 + rows / 2, r0 + rows, r0 + rows + 9, (1 << 23) + 1, most}) {
            if (begin < 0 || begin > end || end > most) continue;
            const RowRange all{begin, end}, got = tiles_within(all, r0, r0 + rows, group);
            const long long n = (long long)rows * group;
            for (long long t = 0; t * 32 < n; ++t)
              if ((t >= got.begin && t < got.end) != truth(all, r0, n, group, t))
                return printf("group %d, rows %d + %d, all %d to %d: tile %lld\n", group, r0, rows, begin, end, t), 1;
          }
  return 0;
}
"""


def run(tmp_path, source):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O2", "-D_GLIBCXX_ASSERTIONS", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout


def test_tiles_of_rows_that_see_all_of_some_keys(tmp_path):
    run(tmp_path, TILES)


def test_an_eviction_numbers_its_pages_in_32_bits():
    """16 forks of the longest sequence there is list 2^30 pages, and as many again may be those after: refused, with the tables as
    they were.  (Their page tables take 4 GB here.)"""
    pool = chunk.Pool(n_pages=1 << 26, max_seqs=20)
    a = pool.new(1 << 30)
    seqs = [a] + pool.fork(a, 15)
    launches = chunk.info()["launches"]
    assert pool.evict(seqs, [1] * 16, ld=1 << 30, kept=None) == XC_ERR_UNSUPPORTED
    assert chunk.info()["launches"] == launches
    live = ctypes.c_int32()
    assert chunk.lib().xc_pool_info(pool.p, ctypes.byref(live), None, None) == XC_OK and live.value == 1 << 26
    assert all(pool.table(s, 0)[1] == 1 << 30 for s in seqs)
    pool.close()


def test_an_eviction_numbers_its_kept_tokens_in_32_bits():
    pool = chunk.Pool(n_pages=1 << 22, page_tokens=256, max_seqs=4)
    a = pool.new(1 << 30)
    seqs = [a] + pool.fork(a, 1)
    assert pool.evict(seqs, [(1 << 29) + 1, 1 << 29], ld=1 << 30, kept=None) == XC_ERR_UNSUPPORTED
    assert [pool.table(s, 0)[1] for s in seqs] == [1 << 30] * 2
    pool.close()


@pytest.mark.parametrize("new", [1, 70])
def test_attention_needs_no_memory_for_weights(new):
    """Where there is room for all but the partial sums, the rows are set and attended; the weights come once there is room."""
    shape = dict(n_pages=3000, q_heads=8, kv_heads=8, dtype=XC_F32 if new == 1 else XC_BF16)

    def rows():
        pool = chunk.Pool(**shape)
        kids = pool.fork(pool.new(5000), 20)
        assert chunk.lib().xc_seq_extend(pool.p, 20, host.ints(*kids), host.ints(*[new] * 20)) == XC_OK
        return pool, kids

    pool, kids = rows()
    before = chunk.info()["live_bytes"]
    assert pool.set(kids, [new] * 20) == XC_OK
    all_of_it = chunk.info()["live_bytes"] - before
    pool.close()
    keys = 128 if new == 1 else 256
    sums = 20 * -(-(5000 + new) // keys) * 8 * keys * 4  # a partial sum per key and head
    pool, kids = rows()
    for room, fits in ((all_of_it - sums // 4 - 1, False), (all_of_it - sums // 4, True)):
        chunk.lib().fake_memory(before + room)
        assert pool.set(kids, [new] * 20) == XC_OK
        assert pool.attention() == XC_OK
        assert pool.weights() == (XC_OK if fits else XC_ERR_OOM) and pool.attention() == XC_OK
    pool.close()
    # asked for again, but not in a capture
    pool, kids = rows()
    chunk.lib().fake_memory(before + all_of_it - sums // 4 - 1)
    assert pool.set(kids, [new] * 20) == XC_OK
    chunk.lib().fake_memory(1 << 60)
    chunk.lib().fake_set(0, 1)
    assert pool.weights() == XC_ERR_OOM and pool.attention() == XC_OK
    chunk.lib().fake_set(0, 0)
    chunk.lib().fake_elsewhere(1)
    assert pool.weights() == XC_OK
    chunk.lib().fake_elsewhere(0)
    chunk.lib().fake_set(0, 1)
    assert pool.weights() == XC_OK and pool.attention() == XC_OK
    chunk.lib().fake_set(0, 0)
    assert chunk.info()["broken_captures"] == 0
    pool.close()
