// Host side of chunks under a mask (xc_chunk_* in include/xcache.h): argument
// validation, what a batch uploads, evictions' tables and the launches.
#include "xc_pool_state.h"

#include <cmath>

using namespace xc;

namespace {

// The batch's partial sums of weights; false: no memory for them.
bool room_for_parts(xc_batch* b) {
  Pool& p = *b->p;
  return enlarge(p, b->parts, b->parts_bytes, b->parts_need, b->parts_need / 4) ||
         enlarge(p, b->parts, b->parts_bytes, b->parts_need, 0);
}

xc_status set_chunk(xc_batch* b, int32_t n, const int32_t* seqs, const int32_t* new_tokens, const ChunkMask& mask) {
  Pool& p = *b->p;
  BatchRows r;
  const xc_status s = batch_rows(p, n, seqs, new_tokens, &r);
  if (s != XC_OK) return s;
  const int n_rows = (int)r.seqs.size(), shift = p.book.shift();
  std::vector<ChunkSeq> chunk_seqs;
  for (int i = 0; i < n_rows; ++i) {
    const PlanSeq& q = r.seqs[i];
    chunk_seqs.push_back({r.first_row[i], q.rows, q.first, q.tokens, q.table, r.number[i]});
  }
  const int group = p.cfg.q_heads / p.cfg.kv_heads;
  const PlanShape shape{group, p.cfg.kv_heads, p.cfg.head_dim, p.esz, p.cus};
  ChunkPlan plan = plan_chunk(chunk_seqs, mask, r.shared_end, shape);
  const long long rows = r.rows;
  auto launches = [&] {  // a launch takes fewer than 2^32 threads
    const long long threads = std::max(((long long)plan.units.size() * p.cfg.kv_heads + kXcds * kXcds) * 512,
                                       plan.n_slots ? rows * p.cfg.q_heads * (p.cfg.head_dim / 4) : 0);
    return threads >> 32 == 0;
  };
  if (!launches()) return XC_ERR_UNSUPPORTED;
  // the sums of weights: where all sequences have few rows, or with partial sums
  int groups = 0;
  const std::vector<WeightRun> runs = plan_weight_runs(chunk_seqs, r.shared_end, shape, &groups);
  std::vector<WeightFew> few;
  std::vector<WeightInfo> infos;
  WeightPlan sums;
  if (p.esz == 2 && !runs.empty()) few = few_runs(runs, chunk_seqs, mask, group, &infos);
  else sums = plan_weights(chunk_seqs, mask, shape);
  if ((((long long)sums.units.size() + kXcds) * p.cfg.kv_heads + kXcds * kXcds) * 256 >> 32 || (long long)groups * 256 >> 32 ||
      (long long)sums.tiles.size() * 1024 >> 32)
    return XC_ERR_UNSUPPORTED;
  // pieces [slot][row][head][D], then their statistics
  auto stat_rows = [&] { return (size_t)plan.n_slots * (rows - plan.piece_row0) * p.cfg.q_heads; };
  auto stats_at = [&] { return align256(stat_rows() * p.cfg.head_dim * sizeof(float)); };
  const size_t piece_need = plan.n_slots ? stats_at() + stat_rows() * sizeof(float2) : 0;
  if (!enlarge(p, b->pieces, b->piece_bytes, piece_need, piece_need / 4)) {
    plan = plan_chunk(chunk_seqs, mask, r.shared_end, shape, 0);  // no memory: without pieces
    if (!launches()) return XC_ERR_OOM;
  }
  std::vector<BatchSeq> batch_seqs;
  for (const PlanPart& part : plan.parts) {
    const ChunkSeq& q = chunk_seqs[part.seq];
    batch_seqs.push_back({part.tok0, q.first + q.tokens - q.rows + (part.tok0 - q.row0), q.table, part.own});
  }
  // uploaded: tables, sequences, units; written on the device: places, own slots
  const size_t o_seqs = align256(r.tables.size() * sizeof(int));
  const size_t o_chunks = o_seqs + align256(batch_seqs.size() * sizeof(BatchSeq));
  const size_t o_units = o_chunks + align256(chunk_seqs.size() * sizeof(ChunkSeq));
  const size_t o_runs = o_units + align256(plan.units.size() * sizeof(ChunkUnit));
  const size_t o_infos = o_runs + align256(few.size() * sizeof(WeightFew));
  const size_t o_sums = o_infos + align256(infos.size() * sizeof(WeightInfo));
  const size_t o_tiles = o_sums + align256(sums.units.size() * sizeof(WeightUnit));
  const size_t up = o_tiles + align256(sums.tiles.size() * sizeof(WeightTile));
  const size_t o_own = up + align256(rows * sizeof(int));
  const size_t need = o_own + align256(rows * sizeof(OwnSlots));
  std::vector<int> seq_copy(seqs, seqs + n);
  // (a quarter more than needed, as of pieces and sums)
  if (!enlarge(p, b->dev, b->dev_bytes, need, need / 4) || !staging(b, b->dev, b->dev_bytes, need, up)) return XC_ERR_OOM;
  // Asked for here, since xc_chunk_weights may be captured; the attention does without.
  b->parts_need = (size_t)sums.parts * p.cfg.kv_heads * (p.esz == 2 ? kWeightKeys : kWeightKeysF32) * sizeof(float);
  (void)room_for_parts(b);
  if (rows > 0) {
    put(b, 0, r.tables);
    put(b, o_seqs, batch_seqs);
    put(b, o_chunks, chunk_seqs);
    put(b, o_units, plan.units);
    put(b, o_runs, few);
    put(b, o_infos, infos);
    put(b, o_sums, sums.units);
    put(b, o_tiles, sums.tiles);
    upload(b, b->dev, up);
    XC_HIP(launch_batch_rows((const int*)b->dev, (const BatchSeq*)(b->dev + o_seqs), (int)batch_seqs.size(), r.rows, shift,
                             (int*)(b->dev + up), (OwnSlots*)(b->dev + o_own), p.st));
  }
  AttnArgs& a = b->attn;
  a = {};
  a.tables = (const int*)b->dev;
  a.chunk_units = (const ChunkUnit*)(b->dev + o_units);
  a.chunk_seqs = (const ChunkSeq*)(b->dev + o_chunks);
  a.mask = mask;
  a.n_units = (int)plan.units.size();
  a.n_long = long_units(plan.units);
  a.group = group;
  a.pieces = (float*)b->pieces;
  a.stats = (float2*)(b->pieces + stats_at());
  a.own = (const OwnSlots*)(b->dev + o_own);
  a.shared_slots = plan.shared_slots;
  a.rows = r.rows;
  a.q_heads = p.cfg.q_heads;
  a.n_slots = plan.n_slots;
  a.piece_row0 = plan.piece_row0;
  a.piece_rows = r.rows - plan.piece_row0;
  a.few = plan.few;
  WeightArgs& w = b->weights;
  w = {};
  w.tables = a.tables;
  w.seqs = a.chunk_seqs;
  w.mask = mask;
  w.q_heads = p.cfg.q_heads;
  w.group = group;
  w.by_group = group == 1 ? 0 : (unsigned)(((1ull << 32) + group - 1) / group);
  w.units = (const WeightUnit*)(b->dev + o_sums);
  w.tiles = (const WeightTile*)(b->dev + o_tiles);
  w.n_units = (int)sums.units.size();
  w.n_long = long_units(sums.units);
  w.n_tiles = (int)sums.tiles.size();
  w.runs = (const WeightFew*)(b->dev + o_runs);
  w.infos = (const WeightInfo*)(b->dev + o_infos);
  w.n_runs = (int)few.size();
  w.n_groups = few.empty() ? 0 : groups;
  b->place = (const int*)(b->dev + up);
  b->rows = r.rows;
  b->seqs.swap(seq_copy);
  b->versions.swap(r.versions);
  b->written.swap(r.written);
  b->chunk = b->set = true;
  return XC_OK;
}

// 0: not a scale
float log2_scale(float scale, int head_dim) {
  const float s = (scale == 0.f ? 1.0f / std::sqrt((float)head_dim) : scale) * 1.4426950408889634f;
  return scale >= 0.f && std::isnormal(s) ? s : 0.f;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// rows of a caller's buffer of pitch ld that start a row each
bool stride_ok(long long ld, long long width, int esz) { return ld >= width && ld <= kMaxStride && ld * esz % 16 == 0; }

}  // namespace

extern "C" {

xc_status xc_chunk_set(xc_batch* b, int32_t n, const int32_t* seqs, const int32_t* new_tokens, const xc_chunk_mask* mask) {
  if (!b || n < 0 || (n > 0 && (!seqs || !new_tokens))) return XC_ERR_INVALID_ARG;
  if (mask && (mask->group < 0 || mask->window < 0 || mask->sinks < 0)) return XC_ERR_INVALID_ARG;
  ChunkMask m{ChunkMask::kNone, ChunkMask::kNone, 0};
  if (mask && mask->group > 0) m.group = mask->group;
  if (mask && mask->window > 0) m.window = mask->window, m.sinks = mask->sinks;
  const xc_status s = guarded(*b->p, [&]() -> xc_status {
    if (!b->p->book.distinct(n, seqs)) return XC_ERR_INVALID_ARG;
    if (capturing(b->p->st)) return XC_ERR_STATE;
    const OutsideCapture outside;
    return set_chunk(b, n, seqs, new_tokens, m);
  });
  if (s == XC_ERR_OOM || s == XC_ERR_HIP) b->set = false, b->rows = 0;  // wherever it failed
  return s;
}

xc_status xc_chunk_attention(xc_batch* b, int32_t block, const void* q, int64_t q_ld, float scale, void* out,
                             int64_t out_ld, float* lse) {
  if (!b || (b->rows > 0 && (!q || !out))) return XC_ERR_INVALID_ARG;
  Pool& p = *b->p;
  const xc_pool_config& c = p.cfg;
  const long long width = (long long)c.q_heads * c.head_dim;
  if (block < 0 || block >= c.n_blocks || !stride_ok(q_ld, width, p.esz) || !stride_ok(out_ld, width, p.esz) ||
      !aligned16(q) || !aligned16(out) || !aligned4(lse))
    return XC_ERR_INVALID_ARG;
  const float s = log2_scale(scale, c.head_dim);
  if (s == 0.f) return XC_ERR_INVALID_ARG;
  return guarded(p, [&]() -> xc_status {
    if (!b->current() || !b->chunk) return XC_ERR_STATE;
    const Rows in = rows_at(q, b->rows, q_ld, width, p.esz), to = rows_at(out, b->rows, out_ld, width, p.esz),
               sums = rows_at(lse, lse ? b->rows : 0, c.q_heads, c.q_heads, 4);
    if (overlap(in, to) || overlap(in, sums) || overlap(to, sums) || p.holds(out, to.extent) || p.holds(lse, sums.extent))
      return XC_ERR_INVALID_ARG;
    if (b->rows == 0) return XC_OK;
    AttnArgs a = b->attn;
    a.buf = p.block(block);
    a.q = q;
    a.q_ld = q_ld;
    a.out = out;
    a.out_ld = out_ld;
    a.scale = s;
    a.lse = lse;
    XC_HIP(launch_branch_attention(c.dtype, a, p.st));
    return XC_OK;
  });
}

xc_status xc_chunk_weights(xc_batch* b, int32_t block, const void* q, int64_t q_ld, float scale, const float* lse,
                           float decay, float* weights, int64_t ld) {
  if (!b || (b->rows > 0 && (!q || !lse || !weights))) return XC_ERR_INVALID_ARG;
  Pool& p = *b->p;
  const xc_pool_config& c = p.cfg;
  const long long width = (long long)c.q_heads * c.head_dim;
  if (block < 0 || block >= c.n_blocks || !stride_ok(q_ld, width, p.esz) || !aligned16(q) || !aligned4(lse) ||
      !aligned4(weights) || ld < 0 || ld > kMaxStride || !(decay >= 0.f) || !std::isfinite(decay))
    return XC_ERR_INVALID_ARG;
  const float s = log2_scale(scale, c.head_dim);
  if (s == 0.f) return XC_ERR_INVALID_ARG;
  return guarded(p, [&]() -> xc_status {
    if (!b->current() || !b->chunk) return XC_ERR_STATE;
    if (q_ld * p.esz >> 28) return XC_ERR_UNSUPPORTED;  // 8 rows within 32 bits
    if (b->rows == 0) return XC_OK;
    int most = 0;
    for (int seq : b->seqs) most = std::max(most, p.book.seq(seq).tokens);
    if (ld < most) return XC_ERR_INVALID_ARG;
    const Rows in = rows_at(q, b->rows, q_ld, width, p.esz), sums = rows_at(lse, b->rows, c.q_heads, c.q_heads, 4),
               to = rows_at(weights, (long long)b->seqs.size(), ld, most, 4);
    if (overlap(in, to) || overlap(sums, to) || p.holds(weights, to.extent)) return XC_ERR_INVALID_ARG;
    if (b->parts_bytes < b->parts_need) {
      if (capturing(p.st)) return XC_ERR_OOM;
      const OutsideCapture outside;
      if (!room_for_parts(b)) return XC_ERR_OOM;
    }
    WeightArgs a = b->weights;
    a.parts = (float*)b->parts;
    a.buf = p.block(block);
    a.q = q;
    a.q_ld = q_ld;
    a.scale = s;
    a.lse = lse;
    a.decay = decay;
    a.weights = weights;
    a.ld = ld;
    XC_HIP(launch_weights(c.dtype, a, p.st));
    return XC_OK;
  });
}

xc_status xc_chunk_evict(xc_batch* b, int32_t n, const int32_t* seqs, const int32_t* keep, int32_t sinks, int32_t recent,
                         float* weights, int64_t ld, int32_t* kept, int64_t kept_ld) {
  if (!b || n < 0 || (n > 0 && (!seqs || !keep)) || sinks < 0 || recent < 0 || !aligned4(weights) || !aligned4(kept) ||
      ld < 0 || ld > kMaxStride || kept_ld < 0 || kept_ld > kMaxStride)
    return XC_ERR_INVALID_ARG;
  Pool& p = *b->p;
  return guarded(p, [&]() -> xc_status {
    if (!p.book.distinct(n, seqs)) return XC_ERR_INVALID_ARG;
    if (capturing(p.st)) return XC_ERR_STATE;
    const OutsideCapture outside;
    std::vector<EvictSeq> list;
    std::vector<int> tables;
    int most_tokens = 0, most_listed = 0, most_kept = 0;
    long long places = 0, pages = 0;
    // the kernels number the pages before and after, which are no more, in 32 bits
    for (int i = 0; i < n; ++i) pages += keep[i] < p.book.seq(seqs[i]).tokens ? p.book.seq(seqs[i]).pages.size() : 0;
    if (pages >= kMaxPlaces) return XC_ERR_UNSUPPORTED;
    for (int i = 0; i < n; ++i) {
      const PageSeq& q = p.book.seq(seqs[i]);
      if (keep[i] < 0) return XC_ERR_INVALID_ARG;
      const bool less = keep[i] < q.tokens;
      if (less && (long long)sinks + recent > keep[i]) return XC_ERR_INVALID_ARG;
      if (q.tokens == 0) continue;
      most_listed = std::max(most_listed, std::min(keep[i], q.tokens));
      if (less) {
        most_tokens = std::max(most_tokens, q.tokens);
        most_kept = std::max(most_kept, keep[i]);
        if (places + keep[i] > kMaxPlaces) return XC_ERR_UNSUPPORTED;
        list.push_back({i, q.first, q.tokens, keep[i], (int)tables.size(), 0, (int)places, 0});
        tables.insert(tables.end(), q.pages.begin(), q.pages.end());
        places += keep[i];
      } else if (kept) {
        list.push_back({i, q.first, q.tokens, -1, 0, 0, 0, 0});
      }
    }
    if (most_tokens > 0 && (!weights || ld < most_tokens)) return XC_ERR_INVALID_ARG;
    if (kept && kept_ld < most_listed) return XC_ERR_INVALID_ARG;
    const Rows w = rows_at(weights, most_tokens ? n : 0, ld, most_tokens, 4),
               k = rows_at(kept, kept ? n : 0, kept_ld, most_listed, 4);
    if (overlap(w, k) || p.holds(weights, w.extent) || p.holds(kept, k.extent)) return XC_ERR_INVALID_ARG;
    if (list.empty()) return XC_OK;
    if (list.size() > 65535) return XC_ERR_UNSUPPORTED;
    // room for twice the tables: the new ones are no longer
    const size_t o_tables = align256(list.size() * sizeof(EvictSeq));
    const size_t up_most = o_tables + align256(2 * tables.size() * sizeof(int));
    const size_t o_stays = up_most + align256((size_t)places * sizeof(int));
    const size_t need = o_stays + align256(list.size() * sizeof(int));
    tables.reserve(2 * tables.size());
    // A few tables go with the launch: nothing to wait for, and no copy.  2304 tokens back to 1536, 8 blocks, 8 heads of 64:
    // 14.5 us a call so, 17.4 with a launch for them alone, 19.8 with a copy; 12 sequences, 20 blocks, 12 heads of 128: 390,
    // 392 and 395.
    Little words{};
    const bool little = up_most <= Little::kMost;
    if (!(little ? enlarge(p, b->evict, b->evict_bytes, need, need / 2) : staging(b, b->evict, b->evict_bytes, need, up_most)))
      return XC_ERR_OOM;
    std::vector<std::vector<int>> next;
    const PageStatus s = p.book.evict(n, seqs, keep, sinks, &next);
    if (s != PageStatus::ok) return status_of(s);
    committed([&] {
      for (EvictSeq& e : list) {
        e.to = (int)tables.size();
        if (e.keep < 0) continue;
        const std::vector<int>& now = next[e.number];
        e.replaced = !std::equal(now.begin(), now.end(), tables.begin() + e.from);
        tables.insert(tables.end(), now.begin(), now.end());
      }
      char* to = little ? words.bytes : b->pinned;
      std::memcpy(to, list.data(), list.size() * sizeof(EvictSeq));
      if (!tables.empty()) std::memcpy(to + o_tables, tables.data(), tables.size() * sizeof(int));
      if (!little) upload(b, b->evict, up_most);
      EvictArgs a{};
      a.seqs = (EvictSeq*)b->evict;
      a.tables = (int*)(b->evict + o_tables);
      a.src = (int*)(b->evict + up_most);
      a.stays = (int*)(b->evict + o_stays);
      a.n = (int)list.size();
      a.sinks = sinks;
      a.recent = recent;
      a.weights = weights;
      a.ld = ld;
      a.kept = kept;
      a.kept_ld = kept_ld;
      XC_HIP(launch_evict(a, little ? &words : nullptr, p.block(0), p.esz, p.cfg.n_blocks, p.block_elems() * p.esz,
                          most_tokens, most_kept, p.st));
    });
    return XC_OK;
  });
}

}  // extern "C"
