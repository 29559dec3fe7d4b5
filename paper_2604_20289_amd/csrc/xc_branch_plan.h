// How the attention of branching sequences is cut into workgroups: host
// arithmetic without HIP.
#pragma once

#include <algorithm>
#include <cstdint>
#include <unordered_map>
#include <vector>

namespace xc {

// A workgroup's share of the attention: the query rows of `tokens` batch rows
// (each with the query heads of one key head) over the keys at places [lo, hi)
// of one sequence's pages.
struct AttnUnit {
  int tok0, tokens;  // batch rows
  int table;         // the sequence's page table begins at tables[table]
  int lo, hi;
  int slot;          // piece the result goes to; -1: it is the whole result
};

struct PlanSeq {
  int rows;           // batch rows (its last tokens)
  int first, tokens;  // keys: places [first, first + tokens) of its pages
  int table;
};

// Query rows (batch row, query head of the group) of a workgroup of the
// attention kernels: bf16 wide and few, float32.
constexpr int kWideRows = 256, kFewRows = 64, kF32Rows = 32;

struct PlanShape {
  int group;      // query heads per key head
  int kv_heads;
  int D;
  int elem;       // bytes per element
  int cus;
};

struct OwnSlots {
  int first, n;
};

// Batch rows tok0 .. of one sequence whose own pieces are in the same slots.
struct PlanPart {
  int seq, tok0, rows;
  OwnSlots own;
};

struct AttnPlan {
  std::vector<AttnUnit> units;
  std::vector<PlanPart> parts;  // all rows, in order
  int piece_row0 = 0;           // the first row that has pieces
  int shared_slots = 0;       // slots 0 .. shared_slots - 1: pieces of the shared history, of every row
  int n_slots = 0;            // 0: no row has pieces
  bool few = false;           // bf16: units for branch_few_kernel
};

constexpr int kPlanMaxSlots = 96;
constexpr int kXcds = 8;  // each has its own L2
// pieces of a plan at most; a plan without any always exists
constexpr long long kPlanMaxPieceBytes = 4ll << 30;

namespace plan_detail {

inline long long cdiv(long long a, long long b) { return (a + b - 1) / b; }

// keys [lo, hi) in tiles of 64 places from lo rounded down to 16 (a group of
// 16 places lies in one page)
inline int tiles_of(int lo, int hi) { return hi > lo ? (int)cdiv(hi - (lo & ~15), 64) : 0; }

// place where piece i of n begins: whole tiles, as even as they go
inline int cut(int lo, int hi, int n, int i) {
  if (i == 0) return lo;
  if (i == n) return hi;
  return (lo & ~15) + 64 * (int)((long long)tiles_of(lo, hi) * i / n);
}

// What a kernel takes.  A workgroup that has the chip to itself needs tile_us
// for a 64-key tile and start_us for everything besides; `per_cu` of them share
// a CU, and together they go at most as fast as `crowd` of them per CU would
// alone.  Measured at d = 128 / 64: the wide kernel's tile is two phases of its
// waves, 1.3 us alone and 1.85 with every CU busy (the chip's power limits the
// clock) / 0.9 either way; the few kernel's is 32 KB, 0.86 us alone (38 KB/us
// through one workgroup's requests; a quarter more with over 32 rows) and 6.0
// TB/s in all; the float32 kernel's is its products'.  Of the latter two fit on
// a CU at d = 64 and three at 32, but they share the matrix units, and a round
// of 256 that is not full takes as long as a full one: 1, 2, 3 and 4 rounds of 32
// tiles take 47, 81, 122 and 158 us (d = 64), 30, 46, 66 and 88 (32), 320
// workgroups 80 and 46.  So they count as one per CU.
struct Kernel {
  int rows;
  bool few;
  double tile[3], start;  // d = 128, 64, 32
  int per_cu;
  double crowd[3];
  static int at(const PlanShape& s) { return s.D == 128 ? 0 : s.D == 64 ? 1 : 2; }
};
constexpr Kernel kWide{kWideRows, false, {1.3, 0.9, 0}, 5.0, 1, {0.7, 1.0, 0}},
    kFew{kFewRows, true, {0.86, 0.43, 0}, 3.0, 2, {0.62, 0.62, 0}},
    kF32{kF32Rows, false, {2.45, 1.2, 0.67}, 4.0, 1, {1.0, 1.0, 1.0}};
// distinct keys and values all CUs together read from HBM
constexpr double kHbmBytesPerUs = 6.0e6;
// the merge's launch, and its pieces written and read
constexpr double kMergeUs = 5.0, kPieceBytesPerUs = 3.0e6;

// of `rows` rows in blocks of `per`, those of the last `left` blocks; `left` less these
inline long long tail_of(long long rows, int per, long long& left) {
  const long long blocks = cdiv(rows, per), mine = std::min(blocks, left);
  left -= mine;
  return mine == blocks ? rows : mine == 0 ? 0 : rows - (blocks - mine) * per;
}

// Time of workgroups on `places` places, the long ones first, each advancing
// by at most 1 us per us and all together by at most `crowd`: equal shares
// until the next one ends, its place then taken by the next in line.
struct Work {
  struct Kind {
    double us;
    long long n;
  };
  std::vector<Kind> kinds, active;
  void add(long long n, double us) {
    if (n > 0) kinds.push_back({us, n});
  }
  double us(long long places, double crowd) {
    std::sort(kinds.begin(), kinds.end(), [](const Kind& a, const Kind& b) { return a.us > b.us; });
    // running ones by what each has been given (us) when it ends, the next to end in front
    auto later = [](const Kind& a, const Kind& b) { return a.us > b.us; };
    active.clear();
    size_t next = 0;
    long long running = 0;
    double now = 0, given = 0;
    for (;;) {
      while (next < kinds.size() && running < places) {
        const long long n = std::min(kinds[next].n, places - running);
        active.push_back({given + kinds[next].us, n});
        std::push_heap(active.begin(), active.end(), later);
        running += n;
        if ((kinds[next].n -= n) == 0) ++next;
      }
      if (running == 0) return now;
      now += (active.front().us - given) / std::min(1.0, crowd / running);
      given = active.front().us;
      const double slack = std::max(0.05 * kinds.back().us, 0.01 * given);  // those that end so soon after end now
      do {
        std::pop_heap(active.begin(), active.end(), later);
        running -= active.back().n;
        active.pop_back();
      } while (!active.empty() && active.front().us <= given + slack);
    }
  }
};

// Blocks of rows over runs of keys that count as equally long: the full run,
// and what of it is not shared.
struct Like {
  int own_tiles, full_tiles;  // of the longest
  bool tall;                  // blocks of more than 32 query rows
  long long blocks = 0;
  double own_keys = 0, full_keys = 0;  // in all
};
// the same for numbers within 1/16 of each other, exact below 32
inline int scale_of(int x) {
  int shift = 0;
  while (x >> shift >= 32) ++shift;
  return shift << 5 | x >> shift;
}

}  // namespace plan_detail

// shared_end: the place up to which every sequence's pages are the same ones
// (whole pages; 0: nothing shared).
//
// Two ways.  Together: the rows of all sequences are packed into workgroups
// that read the shared history once, the rest is read per sequence, and the
// pieces are merged: few rows per sequence.  Apart: each sequence's rows run
// over its history and its own keys in one go: a sequence whose rows fill
// workgroups by themselves gains nothing by packing.  Either way a long run of
// keys is cut into pieces of about `c` tiles, so that few rows still fill the
// chip.  Workgroups that are whole but leave a last round partly filled have
// the keys of just the last rows cut, as many as that round holds.  The
// cheapest of all by the times above is taken, of those whose pieces take at
// most max_piece_bytes (0: no pieces, each sequence's rows in one go).
//
// Host time: 35 us for 16 branches, 120 us for 64 single tokens behind histories
// of different lengths, 0.7 ms for 4096 (sequences of like length are priced as
// one; one by one 0.9 and 19 ms).
inline AttnPlan plan_attention(const std::vector<PlanSeq>& seqs, int shared_end, const PlanShape& sh,
                               long long max_piece_bytes = kPlanMaxPieceBytes) {
  using namespace plan_detail;
  long long rows = 0;
  for (const PlanSeq& q : seqs) rows += q.rows;
  AttnPlan best;
  if (rows == 0) return best;
  const PlanSeq* head = nullptr;  // any sequence with rows: the shared places are in all of them
  for (const PlanSeq& q : seqs)
    if (q.rows > 0 && head == nullptr) head = &q;
  const double piece_bytes = (double)rows * sh.kv_heads * sh.group * (sh.D * 4 + 8);

  auto slots_of = [](int tiles, int c) { return tiles ? (int)cdiv(tiles, c) : 0; };
  double best_us = 0;
  bool have = false, best_packed = false;
  int best_c = 0, best_tail = 0, best_tail_pieces = 1, per = 0;
  static const int kCuts[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 96, 128, 192, 256, 512, 1024};
  constexpr int kWhole = 1 << 26;
  std::vector<Kernel> kernels{sh.elem == 4 ? kF32 : kWide};
  if (sh.elem == 2 && sh.group <= kFewRows) kernels.push_back(kFew);
  const int dim = Kernel::at(sh);
  for (const Kernel& k : kernels) {
    const int kper = std::max(1, k.rows / sh.group);  // batch rows per workgroup
    const long long places = (long long)k.per_cu * sh.cus;
    auto block = [&](long long r) { return std::min<long long>(r, kper) * sh.group > 32; };
    std::vector<Like> likes;
    std::vector<int> like_of;
    std::unordered_map<uint64_t, int> known;
    long long blocks = 0;
    for (const PlanSeq& q : seqs) {
      const int end = q.first + q.tokens, own_lo = std::max(shared_end, q.first);
      Like l{tiles_of(own_lo, end), tiles_of(q.first, end), block(q.rows)};
      const uint64_t key = (uint64_t)scale_of(l.own_tiles) << 32 | scale_of(l.full_tiles) << 1 | (l.tall ? 1 : 0);
      const int at = known.emplace(key, (int)likes.size()).first->second;
      if (at == (int)likes.size()) likes.push_back(l);
      Like& x = likes[at];
      x.own_tiles = std::max(x.own_tiles, l.own_tiles);
      x.full_tiles = std::max(x.full_tiles, l.full_tiles);
      x.blocks += cdiv(q.rows, kper);
      x.own_keys += std::max(0, end - own_lo);
      x.full_keys += q.tokens;
      like_of.push_back(at);
      blocks += cdiv(q.rows, kper);
    }
    Work w;
    auto add = [&](long long n, int tiles, bool tall, int c) {
      const int s = slots_of(tiles, c);
      if (s > 0) w.add(n * s * sh.kv_heads, (double)tiles / s * k.tile[dim] * (k.few && tall ? 1.25 : 1.0) + k.start);
      return s;
    };
    auto time = [&](double keys) {
      const double t = std::max(w.us(places, k.crowd[dim] * sh.cus), keys * 2 * sh.D * sh.elem * sh.kv_heads / kHbmBytesPerUs);
      w.kinds.clear();
      return t;
    };
    auto take = [&](double us, bool packed, int c, int tail, int pieces) {
      if (have && us >= best_us) return;
      have = true, best_us = us, best_packed = packed, best_c = c, best_tail = tail, best_tail_pieces = pieces;
      per = kper, best.few = k.few;
    };
    int longest = 0;
    for (const Like& l : likes) longest = std::max(longest, l.full_tiles);
    for (const bool packed : {false, true}) {
      if (packed && (shared_end == 0 || seqs.size() < 2)) break;
      const int together = packed ? tiles_of(head->first, shared_end) : 0;
      constexpr size_t kNumCuts = sizeof kCuts / sizeof *kCuts;
      for (size_t i = 0; i <= kNumCuts + 1; ++i) {
        // past the list: as many pieces as the slots hold (histories of millions of tokens), one
        const int c = i < kNumCuts ? kCuts[i] : i == kNumCuts ? (int)cdiv(longest, kPlanMaxSlots - 6) : kWhole;
        if (c != kWhole && c >= longest) continue;  // kWhole is the same
        int most = 0;
        long long groups = packed ? cdiv(rows, kper) * slots_of(together, c) : 0;
        for (const Like& l : likes) {
          const int s = slots_of(packed ? l.own_tiles : l.full_tiles, c);
          most = std::max(most, s);
          groups += l.blocks * s;
        }
        if (c != kWhole && groups * sh.kv_heads > 8 * places) continue;  // rounds enough with longer pieces
        const int slots = packed ? slots_of(together, c) + most : most > 1 ? most : 0;
        if (slots > kPlanMaxSlots || slots * piece_bytes > (double)max_piece_bytes) continue;
        double keys = packed ? shared_end - head->first : 0;
        if (packed) add(cdiv(rows, kper), together, block(rows), c);
        for (const Like& l : likes) {
          add(l.blocks, packed ? l.own_tiles : l.full_tiles, l.tall, c);
          keys += packed ? l.own_keys : l.full_keys;
        }
        take(time(keys) + (slots ? kMergeUs + slots * piece_bytes / kPieceBytesPerUs : 0), packed, c, 0, 1);
      }
    }
    // the last blocks of rows, those past the last full round, in pieces
    const long long over = blocks * sh.kv_heads % places;
    if (blocks * sh.kv_heads <= places || over == 0) continue;
    for (int more = 0; more < 2; ++more)
      for (int pieces : {2, 3, 4, 6, 8}) {
        const long long tail = cdiv(over, sh.kv_heads) + more;
        if (tail >= blocks) continue;
        long long left = tail, tail_rows = 0;
        double keys = 0;
        std::vector<long long> whole;
        for (const Like& l : likes) whole.push_back(l.blocks), keys += l.full_keys;
        for (size_t i = seqs.size(); left > 0;) {
          const long long before = left, r = tail_of(seqs[--i].rows, kper, left);
          const Like& l = likes[like_of[i]];
          whole[like_of[i]] -= before - left;
          add(before - left, l.full_tiles, l.tall, (int)cdiv(l.full_tiles, pieces));
          tail_rows += r;
        }
        for (size_t i = 0; i < likes.size(); ++i) add(whole[i], likes[i].full_tiles, likes[i].tall, kWhole);
        const double bytes = (double)pieces * tail_rows / rows * piece_bytes, t = time(keys);
        if (bytes <= (double)max_piece_bytes)
          take(t + kMergeUs + bytes / kPieceBytesPerUs, false, kWhole, (int)tail, pieces);
      }
  }

  auto emit = [&](const PlanSeq& q, int tok0, long long r, int lo, int hi, int slot0, bool direct, int c) {
    const int n = slots_of(tiles_of(lo, hi), c);
    for (int i = 0; i < n; ++i)
      for (long long t = 0; t < r; t += per)
        best.units.push_back({tok0 + (int)t, (int)std::min<long long>(per, r - t), q.table, cut(lo, hi, n, i),
                              cut(lo, hi, n, i + 1), direct && n == 1 ? -1 : slot0 + i});
    return n;
  };
  if (best_packed) best.shared_slots = best.n_slots = emit(*head, 0, rows, head->first, shared_end, 0, false, best_c);
  // the rows that are cut otherwise, from the last sequence backwards
  std::vector<int> tails(seqs.size());
  long long left = best_tail;
  for (size_t i = seqs.size(); i-- > 0;) tails[i] = (int)tail_of(seqs[i].rows, per, left);
  best.piece_row0 = -1;
  int tok0 = 0;
  for (size_t i = 0; i < seqs.size(); ++i) {
    const PlanSeq& q = seqs[i];
    for (const bool tail : {false, true}) {
      const int r = tail ? tails[i] : q.rows - tails[i];
      if (r == 0) continue;
      const int lo = best_packed ? std::max(shared_end, q.first) : q.first, hi = q.first + q.tokens;
      const int c = tail ? (int)cdiv(tiles_of(lo, hi), best_tail_pieces) : best_c;
      const int n = emit(q, tok0, r, lo, hi, best.shared_slots, !best_packed, c);
      best.parts.push_back({(int)i, tok0, r, {best.shared_slots, !best_packed && n == 1 ? 0 : n}});
      if (best_packed || n > 1) {
        best.n_slots = std::max(best.n_slots, best.shared_slots + n);
        if (best.piece_row0 < 0) best.piece_row0 = tok0;
      }
      tok0 += r;
    }
  }
  best.piece_row0 = std::max(best.piece_row0, 0);
  // the long ones first: what begins last is short
  std::stable_sort(best.units.begin(), best.units.end(),
                   [](const AttnUnit& x, const AttnUnit& y) { return x.hi - x.lo > y.hi - y.lo; });
  return best;
}

// The (key head, unit) pairs of the wide kernel, dealt to the XCDs so that the
// workgroups that run on one of them read the same keys and all have a like
// mixture of long and short ones: the heads in runs, a run to `sharers` XCDs,
// its pairs to these in turn: first the units of over half the longest one's
// length, then the others, either heads outermost.  (With all units of a head
// together, the long ones of the last head began late: 550 tiles' time
// instead of 440 for 28 blocks of 12 heads, 21 of them whole and 7 in thirds.  Runs of pairs as they come,
// where one XCD may get the long ones and the next the short: 63 us instead of
// 50 for 4 heads with 54 long units each and 24 short ones.)
struct XcdDeal {
  int sharers, run;  // XCDs of a run of heads, heads of a run
};
constexpr XcdDeal xcd_deal(int kv_heads) {
  const int runs = (kv_heads & -kv_heads) < kXcds ? (kv_heads & -kv_heads) : kXcds;
  return {kXcds / runs, kv_heads / runs};
}
inline int long_units(const std::vector<AttnUnit>& units) {  // sorted
  int n = 0;
  while (n < (int)units.size() && units[n].hi - units[n].lo > (units[0].hi - units[0].lo) / 2) ++n;
  return n;
}
inline long long xcd_grid(long long n_units, int kv_heads) {
  const XcdDeal d = xcd_deal(kv_heads);
  return (d.run * n_units + d.sharers - 1) / d.sharers * kXcds;
}
// workgroup -> pair; false: none
constexpr bool xcd_pair(int workgroup, int n_units, int n_long, int kv_heads, int& u, int& h) {
  const XcdDeal d = xcd_deal(kv_heads);
  const int x = workgroup % kXcds, i = workgroup / kXcds * d.sharers + x % d.sharers;
  if (i >= d.run * n_units) return false;
  const int first = d.run * n_long, n = i < first ? n_long : n_units - n_long, k = i < first ? i : i - first;
  h = x / d.sharers * d.run + k / n;
  u = (i < first ? 0 : n_long) + k % n;
  return true;
}

}  // namespace xc
