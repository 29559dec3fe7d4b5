"""How the attention of branching sequences is cut into workgroups
(csrc/xc_branch_plan.h), on the CPU: every row meets every key of its
sequence once, whatever way is taken."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import branch_reference as ref  # noqa: E402
from paper_2604_20289_amd import build  # noqa: E402

SHIM = r"""
#include "xc_branch_plan.h"
using namespace xc;
static AttnPlan plan;
extern "C" {
int make(int n, const int* seqs, int shared_end, int group, int kv_heads, int D, int elem, int cus) {
  std::vector<PlanSeq> s;
  for (int i = 0; i < n; ++i) s.push_back({seqs[4 * i], seqs[4 * i + 1], seqs[4 * i + 2], seqs[4 * i + 3]});
  plan = plan_attention(s, shared_end, {group, kv_heads, D, elem, cus});
  return (int)plan.units.size();
}
void info(int* out) { out[0] = plan.shared_slots, out[1] = plan.n_slots, out[2] = plan.few; }
void units(int* out) { for (auto& u : plan.units) for (int v : {u.tok0, u.tokens, u.table, u.lo, u.hi, u.slot}) *out++ = v; }
int grid(int units, int heads) { return (int)xcd_grid(units, heads); }
int pair(int wg, int units, int n_long, int heads) {
  int u = -1, h = -1;
  return xcd_pair(wg, units, n_long, heads, u, h) ? h * units + u : -1;
}
int own(int* out) {  // of every row
  for (auto& p : plan.parts) for (int i = 0; i < p.rows; ++i) *out++ = p.seq, *out++ = p.own.first, *out++ = p.own.n;
  return plan.piece_row0;
}
}
"""


@functools.lru_cache(None)
def lib():
    d = tempfile.mkdtemp(prefix="xc_plan_")
    src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D_GLIBCXX_ASSERTIONS", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    build.CSRC, src, "-o", so], check=True)
    return ctypes.CDLL(so)


def plan(seqs, shared_end, group=1, kv_heads=8, D=128, elem=2, cus=256):
    """seqs: (rows, first, tokens, table)."""
    flat = [v for s in seqs for v in s]
    n = lib().make(len(seqs), (ctypes.c_int * len(flat))(*flat), shared_end, group, kv_heads, D, elem, cus)
    units = np.zeros((n, 6), np.int32)
    info, own = np.zeros(3, np.int32), np.full((sum(s[0] for s in seqs), 3), -1, np.int32)
    lib().units(units.ctypes.data_as(ctypes.c_void_p))
    lib().info(info.ctypes.data_as(ctypes.c_void_p))
    row0 = lib().own(own.ctypes.data_as(ctypes.c_void_p))
    assert (own[:, 0] == np.repeat(np.arange(len(seqs)), [s[0] for s in seqs])).all()
    if info[1] == 0:
        assert row0 == 0
    elif row0:  # rows before it are whole
        assert info[0] == 0 and (own[:row0, 2] == 0).all() and own[row0, 2] > 1
    return units, info[0], info[1], own[:, 1:], 32 if elem == 4 else 64 if info[2] else 256


def check(seqs, shared_end, group, **kw):
    units, shared, n_slots, own, tile_rows = plan(seqs, shared_end, group=group, **kw)
    rows = sum(s[0] for s in seqs)
    first_row = np.cumsum([0] + [s[0] for s in seqs])
    seq_of = np.repeat(np.arange(len(seqs)), [s[0] for s in seqs])
    by_row = [[] for _ in range(rows)]
    for tok0, tokens, table, lo, hi, slot in units.tolist():
        assert tokens >= 1 and tokens * group <= max(tile_rows, group) and hi > lo
        assert -1 <= slot < n_slots
        for t in range(tok0, tok0 + tokens):
            # the shared places are read through any sequence's table, others through its own
            assert table == seqs[seq_of[t]][3] or hi <= shared_end
            by_row[t].append((lo, hi, slot))
    for t, got in enumerate(by_row):
        _, first, n, _ = seqs[seq_of[t]]
        got.sort()
        assert got[0][0] == first and got[-1][1] == first + n
        assert all(a[1] == b[0] for a, b in zip(got, got[1:]))
        slots = [s for _, _, s in got]
        if slots == [-1]:
            assert shared == 0 and own[t][1] == 0
        else:
            o = own[t]
            assert sorted(slots) == list(range(shared)) + list(range(o[0], o[0] + o[1]))
    assert first_row[-1] == rows
    return units, shared, n_slots


@pytest.mark.parametrize("seed", range(40))
def test_every_row_meets_every_key_once(seed):
    rng = random.Random(seed)
    page = rng.choice([16, 32, 64, 128, 256])
    n = rng.choice([1, 2, 3, 9])
    first = rng.randint(0, page - 1)
    pages = rng.choice([0, 1, 3, 200])
    shared_end = pages * page if n > 1 else 0
    if shared_end <= first:
        shared_end = 0
    seqs, table = [], 0
    for _ in range(n):
        end = max(shared_end, first + 1) + rng.choice([0, 1, 7, rng.randint(1, 3000)])
        tokens = end - first
        rows = rng.choice([0, 1, min(tokens, 5), rng.randint(1, tokens)])
        seqs.append((rows, first, tokens, table))
        table += -(-end // page)
    # sequences without rows do not reach the plan
    seqs = [s for s in seqs if s[0]]
    if len(seqs) < 2:
        shared_end = 0
    check(seqs, shared_end, rng.choice([1, 2, 3, 5, 12]), kv_heads=rng.choice([1, 4, 12]),
          D=rng.choice([64, 128]), elem=rng.choice([2, 4]), cus=256)


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 5, 8, 12, 24, 31, 256])
@pytest.mark.parametrize("units,n_long", [(1, 1), (2, 1), (7, 7), (8, 3), (60, 36), (333, 332)])
def test_every_pair_has_one_workgroup(units, n_long, heads):
    """Each (head, unit) once; an XCD (workgroup number modulo 8) has its share of every unit, and few heads."""
    grid = lib().grid(units, heads)
    pairs = np.array([lib().pair(w, units, n_long, heads) for w in range(grid)])
    assert sorted(pairs[pairs >= 0]) == list(range(units * heads))
    assert grid % 8 == 0 and grid - units * heads < 64
    for x in range(8):
        mine = pairs[x::8][pairs[x::8] >= 0]
        for part in (mine[mine % units < n_long], mine[mine % units >= n_long]):
            assert (np.diff(part) > 0).all()  # heads outermost
        late = mine % units >= n_long
        assert (np.diff(late.astype(int)) >= 0).all()  # the long ones first
        assert len(set(mine // units)) <= max(1, heads // min(heads & -heads, 8))


@pytest.mark.parametrize("elem,D,kv,rows,tokens", [(2, 128, 12, [7020] * 4, 21060), (2, 64, 16, [5200, 1, 700, 6000], 9000),
                                                   (4, 128, 8, [900, 1200], 4000), (2, 128, 20, [256 * 14], 9000)])
def test_the_last_rows_fill_the_last_round(elem, D, kv, rows, tokens):
    """Many whole workgroups of a few more than full rounds: only the last blocks of rows are cut."""
    seqs = [(r, 3 * i, tokens + r, 1000 * i) for i, r in enumerate(rows)]
    units, shared, n_slots = check(seqs, 0, 1, kv_heads=kv, D=D, elem=elem)
    per = 32 if elem == 4 else 256
    blocks, cut = sum(-(-r // per) for r in rows), set(units[units[:, 5] >= 0][:, 0])
    whole = set(units[units[:, 5] < 0][:, 0])
    assert shared == 0 and n_slots > 1 and len(whole) + len(cut) == blocks and not whole & cut
    assert 0 < len(cut) <= 256 // kv + 1 and max(whole) < min(cut)  # a round at most, and one block


@pytest.mark.parametrize("case", range(len(ref.LAST_ROUND)))
def test_the_gpu_tests_reach_cut_last_rows(case):
    dtype, d, kv, group, lengths = ref.LAST_ROUND[case]
    seqs = [(n, 0, a + n, 1000 * i) for i, (a, n) in enumerate(lengths)]
    units, shared, n_slots = check(seqs, 0, group, kv_heads=kv, D=d, elem=2 if dtype == torch.bfloat16 else 4)
    assert shared == 0 and n_slots > 1 and (units[:, 5] < 0).any() and (units[:, 5] >= 0).any()


@pytest.mark.parametrize("tokens", [10 ** 6, 2 * 10 ** 7, 2 ** 30 - 1])
def test_histories_of_millions_of_tokens_are_cut(tokens):
    for n, end in ((1, 0), (2, (tokens - 100) // 64 * 64)):
        units, shared, n_slots = check([(1, 0, tokens, 0)] * n, end, 1, kv_heads=1)
        assert 64 <= n_slots <= 96


def test_single_tokens_share_their_history():
    # 16 branches, one row each, behind 14040 tokens: the history in workgroups of all 16 rows
    seqs = [(1, 0, 14016 + 24 + 10 * i, 1000 * i) for i in range(16)]
    units, shared, n_slots = check(seqs, 14016, 1, kv_heads=12)
    assert shared > 1 and n_slots > shared
    wide = units[units[:, 1] == 16]
    assert wide[:, 3].min() == 0 and wide[:, 4].max() == 14016
    # enough workgroups for the chip
    assert len(units) * 12 >= 256


def test_whole_chunks_run_apart():
    # 7020 rows per branch fill workgroups alone: one pass over history and own keys, nothing to merge but for
    # the rows that five rounds of 256 workgroups leave
    seqs = [(7020, 0, 21060, 1000 * i) for i in range(4)]
    units, shared, n_slots = check(seqs, 14016, 1, kv_heads=12)
    assert shared == 0 and (units[:, 5] < 0).sum() >= 256 * 5 // 12 - 2
    assert units[units[:, 5] >= 0][:, 0].min() >= 3 * 7020


def test_one_long_sequence_is_cut():
    units, shared, n_slots = check([(1, 3, 48384, 0)], 0, 1, kv_heads=4)
    assert shared == 0 and n_slots == len(units) > 16


@pytest.mark.parametrize("d", [64, 128])
def test_which_kernel_the_tile_tests_reach(d):
    """The shapes of tests/test_gpu_branches.py: 256 heads run in workgroups of 256 rows over 1 to 12 tiles, one head in
    workgroups of few rows."""
    tiles = {256: set(), 64: set()}
    for kv, group, rows in ((1, 1, 200), (1, 1, 511), (256, 1, 65), (256, 1, 200), (256, 1, 257), (256, 4, 3), (256, 4, 40)):
        for i, more in enumerate((0, 1, 62, 63, 64, 130, 195, 400)):
            units, _, _, _, tile_rows = plan([(rows, (0, 1, 15, 7)[i % 4], rows + more, 0)], 0, group=group, kv_heads=kv, D=d)
            if kv == 1 or rows * group > 64:
                assert tile_rows == (256 if kv == 256 else 64)
            tiles[tile_rows] |= set((-(-(units[:, 4] - (units[:, 3] & ~15)) // 64)).tolist())
    assert tiles[256] >= set(range(1, 9)) and tiles[64] >= {1, 2, 3, 4}


def test_no_rows_no_units():
    units, shared, n_slots, _, _ = plan([], 0)
    assert len(units) == 0 and shared == 0 and n_slots == 0


@pytest.mark.parametrize("branches,rows,history,heads,D,elem", [(1000, 257, 8192, 16, 128, 2), (2000, 100, 8192, 16, 128, 2),
                                                               (2000, 260, 8192, 16, 128, 2), (8192, 64, 8192, 16, 128, 2),
                                                               (20000, 20, 8192, 16, 128, 2), (100000, 160, 8192, 16, 128, 2),
                                                               (3000, 300, 4096, 40, 64, 2), (100000, 30, 4096, 16, 32, 4)])
def test_pieces_of_many_branches_stay_within_their_bound(branches, rows, history, heads, D, elem):
    seqs = [(rows, 0, history + rows, 1000 * i) for i in range(branches)]
    units, shared, n_slots, own, _ = plan(seqs, history, kv_heads=heads, D=D, elem=elem)
    with_pieces = (own[:, 1] > 0).any() or shared > 0
    assert (n_slots > 0) == with_pieces
    first = np.flatnonzero(own[:, 1] > 0)[0] if with_pieces and not shared else 0
    assert int(n_slots) * (branches * rows - int(first)) * heads * (4 * D + 8) <= 4 << 30


def test_which_kernels_the_edge_tests_reach():
    """The shapes of tests/test_gpu_branch_edges.py."""
    for D in (64, 128):
        for rows, kv, n in ((90, 256, 3), (90, 256, 1), (70, 256, 1), (257, 256, 1)):
            assert plan([(rows, 0, 300 + rows, 1000 * i) for i in range(n)], 0, kv_heads=kv, D=D)[4] == 256
        for rows, n in ((21, 3), (7, 3), (3, 3), (21, 1)):
            assert plan([(rows, 3, 297 + rows, 1000 * i) for i in range(n)], 128 if n > 1 else 0, kv_heads=1, D=D)[4] == 64
        assert plan([(90, 3, 297 + 90, 1000 * i) for i in range(3)], 128, kv_heads=256, D=D)[4] == 256
