// Rows under a mask: what each of them sees, and how their work is cut into
// workgroups.  Host arithmetic without HIP.
#pragma once

#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

#include "xc_branch_plan.h"

namespace xc {

// The new tokens of a sequence come in groups; a row sees up to its group's
// last token, of that the last `window` and the sequence's first `sinks`.
// No groups, no window: kNone.
struct ChunkMask {
  static constexpr int kNone = 0x7fffffff;
  int group, window, sinks;
};

// A sequence with rows, its last ones.
struct ChunkSeq {
  int row0, rows;     // batch rows
  int first, tokens;  // its tokens: places [first, first + tokens) of its pages
  int table;          // its page table begins at tables[table]
  int number;         // among the batch's sequences
};

// Places that a row sees: [first, sink_end) and [begin, end); sink_end <= end.
struct Seen {
  int begin, end, sink_end;
};
// ... row r of the sequence
constexpr Seen seen(const ChunkSeq& q, const ChunkMask& m, int r) {
  // r < 2^24, so (r / group + 1) * group <= max(group, r + group) stays in 32 bits
  const int g = m.group < q.rows ? m.group : q.rows, groups_end = (r / g + 1) * g;
  const int end = q.tokens - q.rows + (groups_end < q.rows ? groups_end : q.rows);
  const int begin = end > m.window ? end - m.window : 0, sinks = m.sinks < end ? m.sinks : end;
  return {q.first + begin, q.first + end, q.first + sinks};
}

// A workgroup's share of the attention, as AttnUnit, in tiles of 64 places from
// lo rounded down to 16 on, `skip` places left out before tile skip_at (between
// the first tokens and a window).
struct ChunkUnit : AttnUnit {
  int seq;             // sequence of its rows; -1: a shared history, of which every row sees [lo, sink_end) and from
  int from, sink_end;  // place `from` on
  int tiles;
  int skip_at, skip;
  int free_lo, free_n;  // of the tiles from free_lo on, every row sees all of free_n
};

struct ChunkPlan {
  std::vector<ChunkUnit> units;  // the long ones first
  std::vector<PlanPart> parts;   // all rows, in order
  int piece_row0 = 0;            // the first row that has pieces
  int shared_slots = 0;          // slots 0 .. shared_slots - 1: pieces of the shared history, of every row
  int n_slots = 0;               // 0: no row has pieces
  bool few = false;              // bf16: units for the kernel of few rows
};

namespace plan_detail {

// Tiles over places [lo, hi); those from free_lo to free_hi hide nothing from any row.
struct TileRun {
  int lo, hi, tiles = 0, skip_at = 0, skip = 0, free_lo = 0, free_hi = 0;
  int at(int j) const { return (lo & ~15) + 64 * j + (j >= skip_at ? skip : 0); }
  // every row sees places [all_lo, all_hi), and before them and behind them there is no tile of which all rows see all
  void free_between(int all_lo, int all_hi) {
    tiles = std::max(0, (int)cdiv(hi - skip - (lo & ~15), 64));
    const int main = (lo & ~15) + skip;  // where tile 0 would be without the places left out
    free_lo = std::max(skip_at, (int)cdiv(std::max(0, all_lo - main), 64));
    free_hi = std::max(free_lo, std::min(tiles, (std::max(main, all_hi) - main) / 64));
  }
};
// ... of what rows [r0, r1) of a sequence see, from place `from` on (0: all)
inline TileRun tile_run(const ChunkSeq& q, const ChunkMask& m, int r0, int r1, int from) {
  const Seen a = seen(q, m, r0), b = seen(q, m, r1 - 1);
  TileRun t{std::max(q.first, from), b.end};
  const int base = t.lo & ~15, sink_tiles = tiles_of(t.lo, b.sink_end), gap_lo = base + 64 * sink_tiles, gap_hi = a.begin & ~15;
  const int all_lo = std::max(t.lo, b.begin);
  if (gap_hi > gap_lo) {
    if (sink_tiles > 0) t.skip_at = sink_tiles, t.skip = gap_hi - gap_lo;
    else t.lo = a.begin;
  }
  t.free_between(all_lo, a.end);
  return t;
}

}  // namespace plan_detail

// What every row of a batch sees of the places up to shared_end, whose pages
// are the same in all its sequences: [first, sink_end) and [from, to).
struct SharedRun {
  int first, sink_end, from, to;
  bool any() const { return to > from; }
  plan_detail::TileRun run() const {
    plan_detail::TileRun t{sink_end > first || from == first ? first : from, to};
    if (sink_end > first) {
      const int sink_tiles = plan_detail::tiles_of(first, sink_end), gap_lo = (first & ~15) + 64 * sink_tiles;
      if (from > gap_lo) t.skip_at = sink_tiles, t.skip = from - gap_lo;
    }
    t.free_between(from, to);
    return t;
  }
};
inline SharedRun shared_run(const std::vector<ChunkSeq>& seqs, const ChunkMask& mask, int shared_end) {
  SharedRun s{0, 0, 0, 0};
  if (seqs.size() < 2 || shared_end == 0) return s;
  const bool window = mask.window != ChunkMask::kNone;
  s.first = s.from = s.sink_end = seqs[0].first;
  s.to = shared_end;
  int begin = shared_end;
  for (const ChunkSeq& q : seqs) {
    const Seen a = seen(q, mask, 0), b = seen(q, mask, q.rows - 1);
    s.from = std::max(s.from, b.begin);
    s.to = std::min(s.to, a.end);
    begin = std::min(begin, a.begin);
    if (window) s.sink_end = std::max(s.sink_end, b.sink_end);
  }
  s.to &= ~15;
  if (s.from > s.first) s.from = (s.from + 15) & ~15;
  if (window && begin < s.sink_end) s.to = 0;  // windows that reach into the first tokens
  return s;
}

// As plan_attention, for rows under a mask: the same kernels with the same
// times, blocks of rows of unequal length.  shared_end: the place up to which
// every sequence's pages are the same.
inline ChunkPlan plan_chunk(const std::vector<ChunkSeq>& seqs, const ChunkMask& mask, int shared_end, const PlanShape& sh,
                            long long max_piece_bytes = kPlanMaxPieceBytes) {
  using namespace plan_detail;
  ChunkPlan best;
  long long rows = 0;
  for (const ChunkSeq& q : seqs) rows += q.rows;
  if (rows == 0) return best;
  const SharedRun shared = shared_run(seqs, mask, shared_end);
  const TileRun shared_tiles = shared.run();
  // what rows [r0, r1) of a sequence see besides a shared history: before it and behind it
  auto before = [&](const ChunkSeq& q, int r0, int r1) {
    TileRun t{seen(q, mask, r0).begin, shared.from};
    if (t.hi > t.lo) t.free_between(seen(q, mask, r1 - 1).begin, shared.from);
    return t;
  };
  auto behind = [&](const ChunkSeq& q, int r0, int r1) { return tile_run(q, mask, r0, r1, shared.to); };
  const double row_bytes = (double)sh.kv_heads * sh.group * (sh.D * 4 + 8);

  struct Like {
    int tiles;  // of the longest
    bool tall, front;
    long long blocks = 0;
  };
  auto slots_of = [](int tiles, int c) { return tiles ? (int)cdiv(tiles, c) : 0; };
  static const int kCuts[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 96, 128, 192, 256, 512, 1024};
  constexpr size_t kNumCuts = sizeof kCuts / sizeof *kCuts;
  constexpr int kWhole = 1 << 26;
  bool have = false, best_packed = false;
  double best_us = 0;
  int best_c = 0, best_tail = 0, best_pieces = 1, per = 0;
  std::vector<Kernel> kernels{sh.elem == 4 ? kF32 : kWide};
  if (sh.elem == 2 && sh.group <= kFewRows) kernels.push_back(kFew);
  const int dim = Kernel::at(sh);
  int most_rows = 0;
  for (const ChunkSeq& q : seqs) most_rows = std::max(most_rows, q.rows);
  for (const Kernel& k : kernels) {
    const int kper = std::max(1, k.rows / sh.group);
    if (k.few && have && most_rows > 64 * kper) continue;  // (whole chunks: many workgroups to price, and never the cheaper)
    const long long places = (long long)k.per_cu * sh.cus;
    for (const bool packed : {false, true}) {
      if (packed && !shared.any()) break;
      std::vector<Like> likes;
      std::vector<int> like_of;  // of the blocks
      std::unordered_map<uint64_t, int> known;
      double keys = packed ? shared_tiles.tiles * 64 : 0;
      int longest = packed ? shared_tiles.tiles : 0;
      auto count = [&](const TileRun& t, bool tall, bool front) {
        const uint64_t key = (uint64_t)scale_of(t.tiles) << 2 | (tall ? 2 : 0) | (front ? 1 : 0);
        const int at = known.emplace(key, (int)likes.size()).first->second;
        if (at == (int)likes.size()) likes.push_back({t.tiles, tall, front});
        likes[at].tiles = std::max(likes[at].tiles, t.tiles);
        ++likes[at].blocks;
        longest = std::max(longest, t.tiles);
        return at;
      };
      for (const ChunkSeq& q : seqs) {
        int seq_tiles = 0;
        for (int r = 0; r < q.rows; r += kper) {
          const int r1 = std::min(q.rows, r + kper);
          const bool tall = (r1 - r) * sh.group > 32;
          const TileRun t = packed ? behind(q, r, r1) : tile_run(q, mask, r, r1, 0);
          int tiles = t.tiles;
          like_of.push_back(count(t, tall, false));
          if (packed && shared.from > shared.first) {
            const TileRun f = before(q, r, r1);
            count(f, tall, true);
            tiles += f.tiles;
          }
          seq_tiles = std::max(seq_tiles, tiles);
        }
        keys += seq_tiles * 64;
      }
      const int together = packed ? shared_tiles.tiles : 0;
      const long long blocks = (long long)like_of.size(), shared_blocks = packed ? cdiv(rows, kper) : 0;
      Work w;
      auto add = [&](long long n, int tiles, bool tall, int c) {
        const int s = slots_of(tiles, c);
        if (s > 0) w.add(n * s * sh.kv_heads, (double)tiles / s * k.tile[dim] * (k.few && tall ? 1.25 : 1.0) + k.start);
      };
      auto time = [&] {
        const double t = std::max(w.us(places, k.crowd[dim] * sh.cus), keys * 2 * sh.D * sh.elem * sh.kv_heads / kHbmBytesPerUs);
        w.kinds.clear();
        return t;
      };
      auto take = [&](double us, int c, int tail, int pieces) {
        if (have && us >= best_us) return;
        have = true, best_us = us, best_packed = packed, best_c = c, best_tail = tail, best_pieces = pieces;
        per = kper, best.few = k.few;
      };
      for (size_t i = 0; i <= kNumCuts + 1; ++i) {
        // past the list: as many pieces as the slots hold, one
        const int c = i < kNumCuts ? kCuts[i] : i == kNumCuts ? (int)cdiv(longest, kPlanMaxSlots / 3 - 2) : kWhole;
        if (c != kWhole && (c == 0 || c >= longest)) continue;  // kWhole is the same
        long long groups = shared_blocks * slots_of(together, c);
        int most_of[2] = {0, 0};
        for (const Like& l : likes) {
          most_of[l.front] = std::max(most_of[l.front], slots_of(l.tiles, c));
          groups += l.blocks * slots_of(l.tiles, c);
        }
        if (c != kWhole && groups * sh.kv_heads > 8 * places) continue;  // rounds enough with longer pieces
        const int most = most_of[0] + most_of[1];
        const int slots = packed ? slots_of(together, c) + most : most > 1 ? most : 0;
        const double bytes = slots * row_bytes * rows;
        if (slots > kPlanMaxSlots || bytes > (double)max_piece_bytes) continue;
        add(shared_blocks, together, std::min<long long>(rows, kper) * sh.group > 32, c);
        for (const Like& l : likes) add(l.blocks, l.tiles, l.tall, c);
        take(time() + (slots ? kMergeUs + bytes / kPieceBytesPerUs : 0), c, 0, 1);
      }
      // the last blocks of rows, those past the last full round, in pieces
      const long long over = blocks * sh.kv_heads % places;
      if (packed || blocks * sh.kv_heads <= places || over == 0) continue;
      for (long long tail : {cdiv(over, sh.kv_heads), cdiv(over, sh.kv_heads) + 1, blocks / 2, blocks * 3 / 4}) {
        if (tail >= blocks || tail == 0) continue;
        std::vector<long long> cut(likes.size());
        for (long long i = blocks - tail; i < blocks; ++i) ++cut[like_of[i]];
        for (int pieces : {2, 3, 4, 6, 8}) {
          const double bytes = (double)pieces * tail * kper * row_bytes;
          if (bytes > (double)max_piece_bytes) continue;
          for (size_t i = 0; i < likes.size(); ++i) {
            const Like& l = likes[i];
            add(cut[i], l.tiles, l.tall, (int)std::max(1ll, cdiv(l.tiles, pieces)));
            add(l.blocks - cut[i], l.tiles, l.tall, kWhole);
          }
          take(time() + kMergeUs + bytes / kPieceBytesPerUs, kWhole, (int)tail, pieces);
        }
      }
    }
  }

  auto emit = [&](const TileRun& t, int seq, int table, int tok0, int n_tok, int slot0, bool direct, int c) {
    const int n = slots_of(t.tiles, c);
    for (int i = 0; i < n; ++i) {
      const int j0 = (int)((long long)t.tiles * i / n), j1 = (int)((long long)t.tiles * (i + 1) / n);
      ChunkUnit u{};
      u.tok0 = tok0, u.tokens = n_tok, u.table = table, u.seq = seq, u.tiles = j1 - j0;
      u.lo = i == 0 ? t.lo : t.at(j0);
      u.hi = i == n - 1 ? t.hi : t.at(j1 - 1) + 64;
      u.slot = direct && n == 1 ? -1 : slot0 + i;
      if (seq < 0) u.from = shared.from, u.sink_end = shared.sink_end;
      if (t.skip > 0 && t.skip_at > j0 && t.skip_at < j1) u.skip_at = t.skip_at - j0, u.skip = t.skip;
      u.free_lo = std::min(std::max(t.free_lo - j0, 0), u.tiles);
      u.free_n = std::max(0, std::min(t.free_hi - j0, u.tiles) - u.free_lo);
      best.units.push_back(u);
    }
    return n;
  };
  if (best_packed) {
    int n = 0;
    for (long long r = 0; r < rows; r += per)
      n = emit(shared_tiles, -1, seqs[0].table, (int)r, (int)std::min<long long>(per, rows - r), 0, false, best_c);
    best.shared_slots = best.n_slots = n;
  }
  long long blocks = 0, block = 0;
  for (const ChunkSeq& q : seqs) blocks += cdiv(q.rows, per);
  best.piece_row0 = -1;
  for (size_t i = 0; i < seqs.size(); ++i) {
    const ChunkSeq& q = seqs[i];
    for (int r = 0; r < q.rows; r += per, ++block) {
      const int r1 = std::min(q.rows, r + per);
      const TileRun t = best_packed ? behind(q, r, r1) : tile_run(q, mask, r, r1, 0);
      const int c = block >= blocks - best_tail ? (int)std::max(1ll, cdiv(t.tiles, best_pieces)) : best_c;
      int n = 0;
      if (best_packed && shared.from > shared.first)
        n = emit(before(q, r, r1), (int)i, q.table, q.row0 + r, r1 - r, best.shared_slots, false, c);
      n += emit(t, (int)i, q.table, q.row0 + r, r1 - r, best.shared_slots + n, !best_packed, c);
      const OwnSlots own{best.shared_slots, !best_packed && n == 1 ? 0 : n};
      if (!best.parts.empty() && best.parts.back().seq == (int)i && best.parts.back().own.n == own.n)
        best.parts.back().rows += r1 - r;
      else best.parts.push_back({(int)i, q.row0 + r, r1 - r, own});
      if (best_packed || n > 1) {
        best.n_slots = std::max(best.n_slots, best.shared_slots + n);
        if (best.piece_row0 < 0) best.piece_row0 = q.row0 + r;
      }
    }
  }
  best.piece_row0 = std::max(best.piece_row0, 0);
  std::stable_sort(best.units.begin(), best.units.end(), [](const ChunkUnit& x, const ChunkUnit& y) { return x.tiles > y.tiles; });
  return best;
}
inline int long_units(const std::vector<ChunkUnit>& units) {  // sorted
  int n = 0;
  while (n < (int)units.size() && units[n].tiles > units[0].tiles / 2) ++n;
  return n;
}

// ---- the weights of keys

struct RowRange {
  int begin, end;
};
// Rows of the sequence that see some, and that see all, of its places [k0, k1):
// both runs of rows, since what a row sees of the places past the first tokens
// moves on with it.
constexpr RowRange rows_seeing_some(const ChunkSeq& q, const ChunkMask& m, int k0, int k1) {
  const long long old = q.first + (long long)q.tokens - q.rows, g = m.group < q.rows ? m.group : q.rows;
  const long long x = k0 - old, y = k1 - old + m.window;  // r sees some: groups_end > x, groups_end < y
  RowRange r{0, q.rows};
  if (x >= q.rows) r.begin = q.rows;
  else if (x >= 0) r.begin = (int)(x / g * g);
  if (k0 - q.first >= m.sinks && y <= q.rows) {
    const long long n = (y + g - 1) / g - 1;
    r.end = n > 0 ? (int)(n * g) : 0;
  }
  if (r.end > q.rows) r.end = q.rows;
  if (r.end < r.begin) r.end = r.begin;
  return r;
}
constexpr RowRange rows_seeing_all(const ChunkSeq& q, const ChunkMask& m, int k0, int k1) {
  const long long old = q.first + (long long)q.tokens - q.rows, g = m.group < q.rows ? m.group : q.rows;
  const long long x = k1 - old, y = k0 - old + m.window;  // r sees all: groups_end >= x, groups_end <= y
  RowRange r{0, q.rows};
  if (x > q.rows) r.begin = q.rows;
  else if (x > 0) r.begin = (int)(((x + g - 1) / g - 1) * g);
  if (k1 - q.first > m.sinks && y < q.rows) r.end = y >= g ? (int)(y / g * g) : 0;
  if (r.end < r.begin) r.end = r.begin;
  return r;
}

// Of a workgroup's rows [r0, r1), `group` query rows each in tiles of 32: the tiles that lie in rows `all`.  (Within its rows
// first: 2^24 of 256 query rows would not fit into 32 bits.)
constexpr RowRange tiles_within(const RowRange& all, int r0, int r1, int group) {
  const int begin = all.begin < r0 ? r0 : all.begin < r1 ? all.begin : r1, end = all.end < r0 ? r0 : all.end < r1 ? all.end : r1;
  return {((begin - r0) * group + 31) >> 5, ((end - r0) * group) >> 5};
}

// Keys of a workgroup, query rows of a stage of its queries.
constexpr int kWeightKeys = 256, kWeightKeysF32 = 128, kWeightRows = 64, kWeightRowsF32 = 32;
// A workgroup's share: what rows [r0, r1) of a sequence give to the keys at
// places [lo, hi); its sums are partial sums number `part`.
struct WeightUnit {
  int seq, lo, hi, r0, r1, part;
};
// Keys whose partial sums are joined: numbers part .. part + parts - 1.
struct WeightTile {
  int seq, lo, hi, part, parts;
};
struct WeightPlan {
  std::vector<WeightUnit> units;  // the long ones first
  std::vector<WeightTile> tiles;  // all keys
  int parts = 0;
};

// Few rows (bf16; a float32 batch has units): the keys of a run of places and the query rows of sequences
// seq0 .. seq0 + n_seqs - 1, at most kWeightFew of them, which all have these
// places.  Its workgroups begin at number `group0`.
constexpr int kWeightFew = 64;
struct WeightRun {
  int seq0, n_seqs, lo, hi, group0;
};
// Key tiles of a wave of the kernel of few rows, waves that share the heads of
// one, keys of a workgroup.
constexpr int few_keys(int D) { return D == 128 ? 32 : 64; }
constexpr int few_head_waves(int kv_heads) { return kv_heads >= 4 ? 4 : kv_heads >= 2 ? 2 : 1; }
constexpr int few_group_keys(int D, int kv_heads) { return few_keys(D) * 4 / few_head_waves(kv_heads); }

// The runs of a batch whose sequences all have few rows; empty: not all do.  A
// shared history is read once for as many sequences as fit.
inline std::vector<WeightRun> plan_weight_runs(const std::vector<ChunkSeq>& seqs, int shared_end, const PlanShape& sh,
                                               int* groups) {
  std::vector<WeightRun> runs;
  *groups = 0;
  for (const ChunkSeq& q : seqs)
    if ((long long)q.rows * sh.group > kWeightFew) return runs;
  const int keys = few_group_keys(sh.D, sh.kv_heads);
  auto add = [&](int seq0, int n, int lo, int hi) {
    if (hi <= lo) return;
    runs.push_back({seq0, n, lo, hi, *groups});
    *groups += (int)plan_detail::cdiv(hi - (lo & ~15), keys);
  };
  for (size_t i = 0; shared_end > 0 && i < seqs.size();) {
    size_t j = i;
    int rows = 0;
    while (j < seqs.size() && rows + seqs[j].rows * sh.group <= kWeightFew) rows += seqs[j++].rows * sh.group;
    add((int)i, (int)(j - i), seqs[i].first, shared_end);
    i = j;
  }
  for (size_t i = 0; i < seqs.size(); ++i)
    add((int)i, 1, std::max(seqs[i].first, shared_end), seqs[i].first + seqs[i].tokens);
  return runs;
}

// A run as its workgroups read it: with the places of its page table, the batch
// rows, and at infos[info] what they need of each row, then of each sequence.
struct alignas(16) WeightFew {
  int group0, lo, hi, table, first;
  int row0, rows, seqs, info;
};
struct alignas(16) WeightInfo {
  int a, b, c;  // a row: places [first, c) and [a, b) that it sees; a sequence: its number, its query rows [b, c) of the run
};
inline std::vector<WeightFew> few_runs(const std::vector<WeightRun>& runs, const std::vector<ChunkSeq>& seqs, const ChunkMask& mask,
                                       int group, std::vector<WeightInfo>* infos) {
  std::vector<WeightFew> out;
  infos->clear();
  for (const WeightRun& r : runs) {
    const ChunkSeq& head = seqs[r.seq0];
    WeightFew f{r.group0, r.lo, r.hi, head.table, head.first, head.row0, 0, r.n_seqs, (int)infos->size()};
    for (int i = 0; i < r.n_seqs; ++i) {
      const ChunkSeq& q = seqs[r.seq0 + i];
      f.rows += q.rows;
      for (int row = 0; row < q.rows; ++row) {
        const Seen s = seen(q, mask, row);
        infos->push_back({s.begin, s.end, s.sink_end});
      }
    }
    for (int i = 0; i < r.n_seqs; ++i) {
      const ChunkSeq& q = seqs[r.seq0 + i];
      infos->push_back({q.number, (q.row0 - head.row0) * group, (q.row0 + q.rows - head.row0) * group});
    }
    out.push_back(f);
  }
  return out;
}

// Rows in runs of as many stages as are cheapest: a workgroup takes stage_us
// for each, with the others of its CU at work, and start_us for its keys, and
// at the end of the launch some of the CUs wait for the last of them, on
// average a third of one's time.  So the last tiles may have shorter runs.
// Measured: 7020 rows, 21060 keys, 12 heads of 128, causal by frames of 2340: whole
// columns of 37 to 110 stages 456 us, runs of up to 56 stages 423, of 28 459; runs
// of 37 439, whole columns and runs of 27 for the last third 420 (18 for it 423,
// 13 430, 36 421).  24192 causal rows, 16 heads of 128: 1182 without and 1168
// with; 13 causal chunks, 16 heads of 64 on 4: 154 and 151.
inline WeightPlan plan_weights(const std::vector<ChunkSeq>& seqs, const ChunkMask& mask, const PlanShape& sh) {
  using namespace plan_detail;
  const bool f32 = sh.elem == 4;
  const int keys = f32 ? kWeightKeysF32 : kWeightKeys, per = f32 ? kWeightRowsF32 : kWeightRows;
  WeightPlan plan;
  struct Rows {
    RowRange r;
    int stages;
  };
  std::vector<Rows> rows;
  std::vector<std::pair<int, long long>> kinds;  // stages, tiles
  std::unordered_map<int, int> known;
  int longest = 0;
  for (size_t i = 0; i < seqs.size(); ++i) {
    const ChunkSeq& q = seqs[i];
    for (int k = 0; k < q.tokens; k += keys) {
      const int lo = q.first + k, hi = q.first + std::min(q.tokens, k + keys);
      const RowRange r = rows_seeing_some(q, mask, lo, hi);
      const int stages = (int)cdiv((long long)(r.end - r.begin) * sh.group, per);
      plan.tiles.push_back({(int)i, lo, hi, 0, 0});
      rows.push_back({r, stages});
      longest = std::max(longest, stages);
      if (stages == 0) continue;
      const int at = known.emplace(scale_of(stages), (int)kinds.size()).first->second;
      if (at == (int)kinds.size()) kinds.push_back({stages, 0});
      kinds[at].first = std::max(kinds[at].first, stages);
      ++kinds[at].second;
    }
  }
  const double stage_us = f32 ? 0.03 * sh.D : sh.D == 128 ? 2.0 : 1.45, start_us = 4.6;
  const double places = 2.0 * sh.cus;
  double best_us = 0;
  int best_c = 0, best_end = 0;
  size_t best_from = 0;  // from this tile on, runs of best_end stages
  static const int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 40, 56, 80, 112, 160, 224, 320, 448, 1024, 4096, 16384, 65536};
  double all = 0;
  for (const auto& k : kinds) all += (double)k.second * k.first;
  for (int c : kCuts) {
    long long groups = 0;
    for (const auto& k : kinds) groups += k.second * cdiv(k.first, c);
    auto one = [&](int c) { return std::min(c, longest) * stage_us * 0.65 + start_us; };  // alone on its CU
    auto us = [&](long long groups, int last) {
      return std::max(one(c), sh.kv_heads * (all * stage_us + groups * start_us) / places) + one(last) / 3;
    };
    auto take = [&](double t, int end, size_t from) {
      if (best_c == 0 || t < best_us) best_us = t, best_c = c, best_end = end, best_from = from;
    };
    take(us(groups, c), c, rows.size());
    // the last tiles, as much work as CUs wait for, in shorter runs
    const int end = std::max(1, std::min(c, longest) / 4);
    double left = one(c) * 0.75 * places / (sh.kv_heads * stage_us);
    size_t from = rows.size();
    if (end < c && left < all / 2) {
      while (left > 0) {
        const int n = rows[--from].stages;
        left -= n;
        groups += cdiv(n, end) - cdiv(n, c);
      }
      take(us(groups, end), end, from);
    }
    if (c >= longest) break;
  }
  for (size_t i = 0; i < plan.tiles.size(); ++i) {
    WeightTile& t = plan.tiles[i];
    const int n = (int)cdiv(rows[i].stages, i < best_from ? best_c : best_end), tokens = rows[i].r.end - rows[i].r.begin;
    t.part = plan.parts;
    for (int j = 0; j < n; ++j) {
      const int a = (int)((long long)tokens * j / n), b = (int)((long long)tokens * (j + 1) / n);
      if (a == b) continue;
      plan.units.push_back({t.seq, t.lo, t.hi, rows[i].r.begin + a, rows[i].r.begin + b, plan.parts++});
    }
    t.parts = plan.parts - t.part;
  }
  std::stable_sort(plan.units.begin(), plan.units.end(),
                   [](const WeightUnit& x, const WeightUnit& y) { return x.r1 - x.r0 > y.r1 - y.r0; });
  return plan;
}
inline int long_units(const std::vector<WeightUnit>& units) {  // sorted
  int n = 0;
  while (n < (int)units.size() && units[n].r1 - units[n].r0 > (units[0].r1 - units[0].r0) / 2) ++n;
  return n;
}

}  // namespace xc
