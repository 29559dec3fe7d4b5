"""How work under a mask is cut (csrc/xc_chunk_plan.h), compiled with the host compiler: thousands of random batches, every
place of every row compared with the mask's definition."""
import shutil
import subprocess

import pytest

from paper_2604_20289_amd import build

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")

CHECK = r"""
#include "xc_chunk_plan.h"
#include <cstdio>
#include <cstdlib>
using namespace xc;

// the mask's definition, apart from seen()
static bool truth(const ChunkSeq& q, const ChunkMask& m, int r, int place) {
  const int j = place - q.first;
  int end = q.tokens;
  if (m.group != ChunkMask::kNone) {
    end = q.tokens - q.rows + (r / m.group + 1) * m.group;
    if (end > q.tokens) end = q.tokens;
  }
  if (j < 0 || j >= end) return false;
  return m.window == ChunkMask::kNone || j >= end - m.window || j < m.sinks;
}

// attention: every place that a row sees is in exactly one of its pieces and in a tile; a tile that hides something from a
// row is masked, as the kernels read it; its pieces are the slots that the merge reads
static int attention(const std::vector<ChunkSeq>& seqs, ChunkMask m, int shared, PlanShape sh, long long mem) {
  const ChunkPlan p = plan_chunk(seqs, m, shared, sh, mem);
  int rows = 0, at = 0;
  for (auto& q : seqs) rows += q.rows;
  const int per = std::max(1, (sh.elem == 4 ? kF32Rows : p.few ? kFewRows : kWideRows) / sh.group);
  std::vector<OwnSlots> own(rows);
  for (auto& x : p.parts) {
    if (x.tok0 != at) return 1;
    for (int i = 0; i < x.rows; ++i) own[at++] = x.own;
  }
  if (at != rows) return 2;
  std::vector<std::vector<char>> cover(rows);
  std::vector<std::vector<int>> slots(rows);
  std::vector<int> seq_of(rows);
  for (size_t i = 0; i < seqs.size(); ++i)
    for (int r = 0; r < seqs[i].rows; ++r) seq_of[seqs[i].row0 + r] = i, cover[seqs[i].row0 + r].assign(seqs[i].tokens, 0);
  int length = 1 << 30;
  for (auto& u : p.units) {
    const int base = u.lo & ~15, n = (u.hi - u.skip - base + 63) / 64;
    if (u.tokens > per || u.tokens < 1 || u.tiles < 1 || n != u.tiles || u.skip % 16 || u.tiles > length) return 3;
    length = u.tiles;  // the long ones first
    for (int k = 0; k < u.tokens; ++k) {
      const int t = u.tok0 + k;
      const ChunkSeq& q = seqs[seq_of[t]];
      if (u.seq >= 0 && u.seq != seq_of[t]) return 4;
      slots[t].push_back(u.slot);
      const Seen w = seen(q, m, t - q.row0);
      int begin, end, sink_end;
      if (u.seq >= 0) begin = std::max(w.begin, u.lo), end = std::min(w.end, u.hi), sink_end = std::min(w.sink_end, u.hi);
      else begin = std::max(u.from, u.lo), end = u.hi, sink_end = std::min(u.sink_end, u.hi);
      for (int j = 0; j < n; ++j) {
        const int a = base + 64 * j + (j * 64 >= u.skip_at * 64 ? u.skip : 0);
        const bool masked = (unsigned)(j - u.free_lo) >= (unsigned)u.free_n;
        for (int x = a; x < a + 64; ++x) {
          const bool s = (x >= begin && x < end) || (x >= u.lo && x < sink_end);
          if (!masked && !s) return 5;
          if (s && !truth(q, m, t - q.row0, x)) return 6;
          if (s && ++cover[t][x - q.first] > 1) return 7;
          if (s && x >= u.hi) return 8;
        }
        // tiles of 32 are halves of these
        for (int e = 0; e < 2; ++e)
          if (base + 32 * (2 * j + e) + ((2 * j + e) * 32 >= u.skip_at * 64 ? u.skip : 0) != a + 32 * e) return 9;
      }
    }
  }
  for (int t = 0; t < rows; ++t) {
    const ChunkSeq& q = seqs[seq_of[t]];
    for (int j = 0; j < q.tokens; ++j)
      if (truth(q, m, t - q.row0, q.first + j) != (cover[t][j] == 1)) return 10;
    std::vector<int> want;
    if (own[t].n == 0 && p.shared_slots == 0) want = {-1};
    for (int i = 0; i < p.shared_slots; ++i) want.push_back(i);
    for (int i = 0; i < own[t].n; ++i) want.push_back(own[t].first + i);
    std::sort(slots[t].begin(), slots[t].end());
    if (slots[t] != want) return 11;
    for (int x : want)
      if (x >= p.n_slots || x >= kPlanMaxSlots || (x >= 0 && t < p.piece_row0)) return 12;
  }
  if (mem == 0 && p.n_slots) return 13;
  return 0;
}

// weights: every (row, key) pair that is seen is in exactly one unit, every key in one tile with its units' sums
static int weights(const std::vector<ChunkSeq>& seqs, ChunkMask m, PlanShape sh) {
  const WeightPlan p = plan_weights(seqs, m, sh);
  const int keys = sh.elem == 4 ? kWeightKeysF32 : kWeightKeys;
  std::vector<const WeightUnit*> by_part(p.parts, nullptr);
  for (auto& u : p.units) {
    if (u.part < 0 || u.part >= p.parts || by_part[u.part] || u.r0 >= u.r1 || u.hi - u.lo > keys || u.lo >= u.hi) return 21;
    if ((long long)(u.r1 - u.r0) * sh.group >= 1 << 23) return 22;
    by_part[u.part] = &u;
  }
  std::vector<std::vector<int>> tile_of(seqs.size());
  for (size_t i = 0; i < seqs.size(); ++i) tile_of[i].assign(seqs[i].tokens, -1);
  for (size_t i = 0; i < p.tiles.size(); ++i)
    for (int x = p.tiles[i].lo; x < p.tiles[i].hi; ++x) {
      int& t = tile_of[p.tiles[i].seq][x - seqs[p.tiles[i].seq].first];
      if (t >= 0) return 23;
      t = i;
    }
  for (size_t i = 0; i < seqs.size(); ++i)
    for (int j = 0; j < seqs[i].tokens; ++j) {
      if (tile_of[i][j] < 0) return 24;
      const WeightTile& t = p.tiles[tile_of[i][j]];
      std::vector<char> rows(seqs[i].rows, 0);
      for (int k = t.part; k < t.part + t.parts; ++k) {
        const WeightUnit* u = by_part[k];
        if (!u || u->seq != (int)i || u->lo != t.lo || u->hi != t.hi) return 25;
        for (int r = u->r0; r < u->r1; ++r)
          if (rows[r]++) return 26;
      }
      for (int r = 0; r < seqs[i].rows; ++r)
        if (truth(seqs[i], m, r, seqs[i].first + j) && !rows[r]) return 27;
    }
  return 0;
}

// few rows: every key of every sequence is in exactly one run that has the sequence
static int runs(const std::vector<ChunkSeq>& seqs, int shared, PlanShape sh) {
  int groups = 0;
  const auto rs = plan_weight_runs(seqs, shared, sh, &groups);
  bool few = true;
  for (auto& q : seqs) few &= q.rows * sh.group <= kWeightFew;
  if (few == rs.empty()) return 31;
  if (!few) return 0;
  std::vector<std::vector<char>> cover(seqs.size());
  for (size_t i = 0; i < seqs.size(); ++i) cover[i].assign(seqs[i].tokens, 0);
  int next = 0;
  for (auto& r : rs) {
    if (r.group0 != next) return 32;
    next += (r.hi - (r.lo & ~15) + few_group_keys(sh.D, sh.kv_heads) - 1) / few_group_keys(sh.D, sh.kv_heads);
    int rows = 0;
    for (int i = r.seq0; i < r.seq0 + r.n_seqs; ++i) {
      rows += seqs[i].rows * sh.group;
      for (int x = r.lo; x < r.hi; ++x)
        if (x < seqs[i].first || cover[i][x - seqs[i].first]++) return 33;
    }
    if (rows > kWeightFew || r.n_seqs > kWeightFew) return 34;
  }
  if (next != groups) return 35;
  for (auto& c : cover)
    for (char x : c)
      if (x != 1) return 36;
  return 0;
}

int main() {
  srand(1);
  int packed = 0, windowed = 0, cut = 0, few = 0, skips = 0, tails = 0;
  for (int it = 0; it < 2500; ++it) {
    const bool single = rand() % 3 == 0;
    const int n = 1 + rand() % (single ? 20 : 5), group = 1 << rand() % 4;
    std::vector<ChunkSeq> s;
    const int pre = rand() % 3 ? rand() % 3000 : 0, page = 16 << rand() % 5, first = rand() % 16;
    const bool sharing = rand() % 2 && n > 1;
    int shared = sharing ? (first + pre) / page * page : 0, row0 = 0;
    for (int i = 0; i < n; ++i) {
      const int rows = rand() % 4 && !single ? 1 + rand() % (rand() % 2 ? 20 : 700) : 1;
      const int tokens = (sharing ? pre : rand() % 2000) + rows + rand() % 100;
      s.push_back({row0, rows, sharing ? first : rand() % 256, tokens, 0, i});
      row0 += rows;
    }
    ChunkMask m{rand() % 3 ? 1 + rand() % (rand() % 2 ? 4 : 300) : ChunkMask::kNone,
                rand() % 2 ? 1 + rand() % (rand() % 2 ? 30 : 1500) : ChunkMask::kNone, 0};
    if (m.window != ChunkMask::kNone && rand() % 2) m.sinks = rand() % 300;
    const PlanShape sh{group, 1 + rand() % 16, rand() % 2 ? 128 : 64, rand() % 4 ? 2 : 4, 256};
    const long long mem = rand() % 5 ? kPlanMaxPieceBytes : 0;
    int bad = attention(s, m, shared, sh, mem);
    if (!bad) bad = weights(s, m, sh);
    if (!bad) bad = runs(s, shared, sh);
    if (bad) return printf("batch %d: %d\n", it, bad), 1;
    const ChunkPlan p = plan_chunk(s, m, shared, sh, mem);
    packed += p.shared_slots > 0;
    windowed += p.shared_slots > 0 && m.window != ChunkMask::kNone;
    cut += p.n_slots > 0;
    few += p.few;
    tails += p.n_slots > 0 && p.shared_slots == 0 && p.piece_row0 > 0;
    for (auto& u : p.units)
      if (u.skip) { ++skips; break; }
  }
  // rows that see all of some keys, as a workgroup of the weights takes it: none of them hides any
  for (int it = 0; it < 100000; ++it) {
    const int rows = 1 + rand() % 60, tokens = rows + rand() % 80;
    const ChunkSeq q{0, rows, rand() % 30, tokens, 0, 0};
    ChunkMask m{rand() % 3 ? 1 + rand() % 70 : ChunkMask::kNone, rand() % 2 ? 1 + rand() % 100 : ChunkMask::kNone, 0};
    if (m.window != ChunkMask::kNone && rand() % 2) m.sinks = rand() % 60;
    const int k0 = q.first + rand() % tokens, k1 = k0 + 1 + rand() % (q.first + tokens - k0);
    const RowRange some = rows_seeing_some(q, m, k0, k1), all = rows_seeing_all(q, m, k0, k1);
    for (int r = 0; r < rows; ++r) {
      bool any = false, every = true;
      for (int x = k0; x < k1; ++x) any |= truth(q, m, r, x), every &= truth(q, m, r, x);
      if (any != (r >= some.begin && r < some.end)) return printf("rows %d: some\n", it), 1;
      if (!every && r >= all.begin && r < all.end) return printf("rows %d: all\n", it), 1;
    }
  }
  // division by the query heads of a group as the kernels do it
  for (unsigned group = 2; group <= 256; ++group) {
    const unsigned by = (unsigned)(((1ull << 32) + group - 1) / group);
    for (unsigned i = 0; i < 1u << 23; i += 1 + rand() % 4096)
      for (unsigned x : {i, i / group * group, i / group * group + group - 1})
        if ((unsigned)(((unsigned long long)x * by) >> 32) != x / group) return printf("group %u: %u\n", group, x), 1;
  }
  printf("%d %d %d %d %d %d\n", packed, windowed, cut, few, skips, tails);
  return 0;
}
"""


def test_plans_of_random_batches(tmp_path):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text(CHECK)
    subprocess.run(["g++", "-std=c++17", "-O2", "-D_GLIBCXX_ASSERTIONS", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
    kinds = [int(x) for x in r.stdout.split()]
    assert all(k > 10 for k in kinds), kinds  # every kind of plan was among them
