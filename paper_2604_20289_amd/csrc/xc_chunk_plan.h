// Rows under a mask: what each of them sees, and how their work is cut into
// workgroups.  Host arithmetic without HIP.
#pragma once

#include <algorithm>
#include <cstdint>
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
  int seq;             // sequence of its rows; -1: a shared history, of which every row sees all
  int tiles;
  int skip_at, skip;
  int all_lo, all_hi;  // every row sees every place of them
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

// The tiles of rows [r0, r1) of a sequence, from place `from` on (0: all they see).
struct TileRun {
  int lo, hi, tiles, skip_at, skip, all_lo, all_hi;
  int at(int j) const { return (lo & ~15) + 64 * j + (j >= skip_at ? skip : 0); }
};
inline TileRun tile_run(const ChunkSeq& q, const ChunkMask& m, int r0, int r1, int from) {
  const Seen a = seen(q, m, r0), b = seen(q, m, r1 - 1);
  TileRun t{std::max(q.first, from), b.end, 0, 0, 0, 0, 0};
  t.all_lo = std::max(t.lo, b.begin);
  t.all_hi = a.end;
  const int gap_lo = b.sink_end > t.lo ? (t.lo & ~15) + 64 * tiles_of(t.lo, b.sink_end) : t.lo & ~15, gap_hi = a.begin & ~15;
  if (gap_hi > gap_lo) {
    if (b.sink_end > t.lo) t.skip_at = (gap_lo - (t.lo & ~15)) / 64, t.skip = gap_hi - gap_lo;
    else t.lo = a.begin;
  }
  t.tiles = std::max(0, (int)cdiv(t.hi - t.skip - (t.lo & ~15), 64));
  return t;
}

}  // namespace plan_detail

// As plan_attention, for rows under a mask: the same kernels with the same
// times, blocks of rows of unequal length.  shared_end: the place up to which
// every sequence's pages are the same.
inline ChunkPlan plan_chunk(const std::vector<ChunkSeq>& seqs, const ChunkMask& mask, int shared_end, const PlanShape& sh,
                            long long max_piece_bytes = kPlanMaxPieceBytes) {
  using namespace plan_detail;
  ChunkPlan best;
  long long rows = 0;
  int wholly = shared_end;  // what every row sees of the shared places
  for (const ChunkSeq& q : seqs) rows += q.rows, wholly = std::min(wholly, seen(q, mask, 0).end);
  if (rows == 0) return best;
  wholly &= ~15;
  if (mask.window != ChunkMask::kNone || seqs.size() < 2 || wholly <= seqs[0].first) wholly = 0;
  const double row_bytes = (double)sh.kv_heads * sh.group * (sh.D * 4 + 8);

  struct Like {
    int tiles;  // of the longest
    bool tall;
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
      if (packed && wholly == 0) break;
      const int from = packed ? wholly : 0;
      std::vector<Like> likes;
      std::vector<int> like_of;  // of the blocks
      std::unordered_map<uint64_t, int> known;
      double keys = packed ? wholly - seqs[0].first : 0;
      int longest = 0;
      for (const ChunkSeq& q : seqs) {
        int seq_keys = 0;
        for (int r = 0; r < q.rows; r += kper) {
          const int r1 = std::min(q.rows, r + kper);
          const TileRun t = tile_run(q, mask, r, r1, from);
          const bool tall = (r1 - r) * sh.group > 32;
          const int at = known.emplace((uint64_t)scale_of(t.tiles) << 1 | (tall ? 1 : 0), (int)likes.size()).first->second;
          if (at == (int)likes.size()) likes.push_back({t.tiles, tall});
          likes[at].tiles = std::max(likes[at].tiles, t.tiles);
          ++likes[at].blocks;
          like_of.push_back(at);
          longest = std::max(longest, t.tiles);
          seq_keys = std::max(seq_keys, t.tiles * 64);
        }
        keys += seq_keys;
      }
      const int together = packed ? tiles_of(seqs[0].first, wholly) : 0;
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
        const int c = i < kNumCuts ? kCuts[i] : i == kNumCuts ? (int)cdiv(std::max(longest, together), kPlanMaxSlots - 6) : kWhole;
        if (c != kWhole && (c == 0 || c >= std::max(longest, together))) continue;  // kWhole is the same
        long long groups = shared_blocks * slots_of(together, c);
        int most = 0;
        for (const Like& l : likes) {
          most = std::max(most, slots_of(l.tiles, c));
          groups += l.blocks * slots_of(l.tiles, c);
        }
        if (c != kWhole && groups * sh.kv_heads > 8 * places) continue;  // rounds enough with longer pieces
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
      for (int more = 0; more < 2; ++more)
        for (int pieces : {2, 3, 4, 6, 8}) {
          const long long tail = cdiv(over, sh.kv_heads) + more;
          if (tail >= blocks) continue;
          const double bytes = (double)pieces * tail * kper * row_bytes;
          if (bytes > (double)max_piece_bytes) continue;
          std::vector<long long> whole;
          for (const Like& l : likes) whole.push_back(l.blocks);
          for (long long i = blocks - tail; i < blocks; ++i) {
            const Like& l = likes[like_of[i]];
            --whole[like_of[i]];
            add(1, l.tiles, l.tall, (int)std::max(1ll, cdiv(l.tiles, pieces)));
          }
          for (size_t i = 0; i < likes.size(); ++i) add(whole[i], likes[i].tiles, likes[i].tall, kWhole);
          take(time() + kMergeUs + bytes / kPieceBytesPerUs, kWhole, (int)tail, pieces);
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
      if (t.skip > 0 && t.skip_at > j0 && t.skip_at < j1) u.skip_at = t.skip_at - j0, u.skip = t.skip;
      u.all_lo = t.all_lo, u.all_hi = t.all_hi;
      best.units.push_back(u);
    }
    return n;
  };
  if (best_packed) {
    TileRun t{seqs[0].first, wholly, tiles_of(seqs[0].first, wholly), 0, 0, seqs[0].first, wholly};
    int n = 0;
    for (long long r = 0; r < rows; r += per)
      n = emit(t, -1, seqs[0].table, (int)r, (int)std::min<long long>(per, rows - r), 0, false, best_c);
    best.shared_slots = best.n_slots = n;
  }
  long long blocks = 0, block = 0;
  for (const ChunkSeq& q : seqs) blocks += cdiv(q.rows, per);
  best.piece_row0 = -1;
  for (size_t i = 0; i < seqs.size(); ++i) {
    const ChunkSeq& q = seqs[i];
    for (int r = 0; r < q.rows; r += per, ++block) {
      const int r1 = std::min(q.rows, r + per);
      const TileRun t = tile_run(q, mask, r, r1, best_packed ? wholly : 0);
      const int c = block >= blocks - best_tail ? (int)std::max(1ll, cdiv(t.tiles, best_pieces)) : best_c;
      const int n = emit(t, (int)i, q.table, q.row0 + r, r1 - r, best.shared_slots, !best_packed, c);
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

}  // namespace xc
