// Host side of the branching cache (xc_pool, xc_batch in include/xcache.h):
// argument validation, page tables, the plan of a batch and the launches.
//
// Device state of a batch: the page tables of its sequences, the attention's
// units and, per row, the place its token has in the pages and the slots of
// its pieces; and the pieces themselves.  Tables go up from pinned memory on
// the pool's stream.  A buffer that became too small goes once the work before
// is done (a graph captured before is not replayed after a new xc_batch_set).
#include "xc_pool_state.h"

#include <cmath>

using namespace xc;

namespace {

constexpr int kMaxHeads = 1024;

void copy_pages(Pool& p, const std::vector<PageCopy>& copies) {
  for (size_t i = 0; i < copies.size(); i += kCopyBatch)
    XC_HIP(launch_page_copies(copies.data() + i, (int)std::min<size_t>(kCopyBatch, copies.size() - i), p.block(0), p.esz,
                              p.cfg.n_blocks, p.block_elems() * p.esz, p.st));
}

RopeFreqs rope_freqs(int d, int axes, double theta) {
  RopeFreqs f{};
  const int d1 = axes == 3 ? 2 * (d / 6) : 0;
  f.axes = axes;
  f.n0 = (d - 2 * d1) / 2;
  f.n1 = d1 / 2;
  for (int i = 0; i < d / 2; ++i) {
    const int np = i < f.n0 ? f.n0 : f.n1, k = i < f.n0 ? i : (i - f.n0) % f.n1;
    f.turns[i] = std::pow(theta, -(double)k / np) / (2.0 * M_PI);
  }
  return f;
}

xc_status set_batch(xc_batch* b, int32_t n, const int32_t* seqs, const int32_t* new_tokens) {
  Pool& p = *b->p;
  const int shift = p.book.shift();
  BatchRows r;
  const xc_status s = batch_rows(p, n, seqs, new_tokens, &r);
  if (s != XC_OK) return s;
  const std::vector<PlanSeq>& plan_seqs = r.seqs;
  const std::vector<int>& tables = r.tables;
  const long long rows = r.rows;
  std::vector<BatchSeq> batch_seqs;
  const int group = p.cfg.q_heads / p.cfg.kv_heads;
  const PlanShape shape{group, p.cfg.kv_heads, p.cfg.head_dim, p.esz, p.cus};
  AttnPlan plan = plan_attention(plan_seqs, r.shared_end, shape);
  auto launches = [&] {  // a launch takes fewer than 2^32 threads
    const long long threads = std::max(((long long)plan.units.size() * p.cfg.kv_heads + kXcds * kXcds) * 512,
                                       plan.n_slots ? rows * p.cfg.q_heads * (p.cfg.head_dim / 4) : 0);
    return threads >> 32 == 0;
  };
  if (!launches()) return XC_ERR_UNSUPPORTED;
  // pieces [slot][row][head][D], then their statistics
  auto stat_rows = [&] { return (size_t)plan.n_slots * (rows - plan.piece_row0) * p.cfg.q_heads; };
  auto stats_at = [&] { return align256(stat_rows() * p.cfg.head_dim * sizeof(float)); };
  const size_t piece_need = plan.n_slots ? stats_at() + stat_rows() * sizeof(float2) : 0;
  if (!enlarge(p, b->pieces, b->piece_bytes, piece_need, piece_need / 4)) {
    plan = plan_attention(plan_seqs, r.shared_end, shape, 0);  // no memory: without pieces
    if (!launches()) return XC_ERR_OOM;
  }
  for (const PlanPart& part : plan.parts) {
    const PlanSeq& q = plan_seqs[part.seq];
    const int at = q.first + q.tokens - q.rows + (part.tok0 - r.first_row[part.seq]);
    batch_seqs.push_back({part.tok0, at, q.table, part.own});
  }

  // uploaded: tables, sequences, units; written on the device: places, own slots
  const size_t o_seqs = align256(tables.size() * sizeof(int));
  const size_t o_units = o_seqs + align256(batch_seqs.size() * sizeof(BatchSeq));
  const size_t up = o_units + align256(plan.units.size() * sizeof(AttnUnit));
  const size_t o_own = up + align256(rows * sizeof(int));
  const size_t need = o_own + align256(rows * sizeof(OwnSlots));
  std::vector<int> seq_copy(seqs, seqs + n);

  if (!staging(b, b->dev, b->dev_bytes, need, up)) return XC_ERR_OOM;
  if (rows > 0) {
    put(b, 0, tables);
    put(b, o_seqs, batch_seqs);
    put(b, o_units, plan.units);
    upload(b, b->dev, up);
    XC_HIP(launch_batch_rows((const int*)b->dev, (const BatchSeq*)(b->dev + o_seqs), (int)batch_seqs.size(), (int)rows,
                             shift, (int*)(b->dev + up), (OwnSlots*)(b->dev + o_own), p.st));
  }
  AttnArgs& a = b->attn;
  a = {};
  a.tables = (const int*)b->dev;
  a.units = (const AttnUnit*)(b->dev + o_units);
  a.n_units = (int)plan.units.size();
  a.n_long = long_units(plan.units);
  a.group = group;
  a.pieces = (float*)b->pieces;
  a.stats = (float2*)(b->pieces + stats_at());
  a.own = (const OwnSlots*)(b->dev + o_own);
  a.shared_slots = plan.shared_slots;
  a.rows = (int)rows;
  a.q_heads = p.cfg.q_heads;
  a.n_slots = plan.n_slots;
  a.piece_row0 = plan.piece_row0;
  a.piece_rows = (int)rows - plan.piece_row0;
  a.few = plan.few;
  b->place = (const int*)(b->dev + up);
  b->rows = (int)rows;
  b->seqs.swap(seq_copy);
  b->versions.swap(r.versions);
  b->written.swap(r.written);
  b->chunk = false;
  b->set = true;
  return XC_OK;
}

}  // namespace

extern "C" {

xc_status xc_pool_init(const xc_pool_config* c, void* keys, void* values, void* hip_stream, xc_pool** out) {
  if (!c || !keys || !values || !out) return XC_ERR_INVALID_ARG;
  *out = nullptr;
  if (c->n_blocks < 1 || c->kv_heads < 1 || c->q_heads < 1 || c->q_heads % c->kv_heads || c->n_pages < 1 ||
      c->max_seqs < 1 || (c->dtype != XC_F32 && c->dtype != XC_BF16) || c->head_dim < 1 || c->page_tokens < 1)
    return XC_ERR_INVALID_ARG;
  int shift = 4;
  while (shift < 8 && (1 << shift) != c->page_tokens) ++shift;
  if ((1 << shift) != c->page_tokens) return XC_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128 && !(c->dtype == XC_F32 && c->head_dim == 32)) return XC_ERR_UNSUPPORTED;
  if (c->q_heads > kMaxHeads || c->q_heads / c->kv_heads > (c->dtype == XC_BF16 ? kWideRows : kF32Rows) || c->n_blocks > 4096 ||
      c->max_seqs > (1 << 20) || (long long)c->n_pages << shift > kMaxPlaces)
    return XC_ERR_UNSUPPORTED;
  if (!aligned16(keys) || !aligned16(values)) return XC_ERR_INVALID_ARG;
  try {
    auto p = std::make_shared<Pool>(*c, shift);
    p->esz = c->dtype == XC_BF16 ? 2 : 4;
    const size_t bytes = (size_t)p->block_elems() * c->n_blocks * p->esz;
    if (overlap(keys, bytes, values, bytes)) return XC_ERR_INVALID_ARG;
    p->keys = (char*)keys;
    p->values = (char*)values;
    p->st = reinterpret_cast<hipStream_t>(hip_stream);
    XC_HIP(hipGetDevice(&p->device));
    XC_HIP(hipDeviceGetAttribute(&p->cus, hipDeviceAttributeMultiprocessorCount, p->device));
    *out = new xc_pool{std::move(p)};
  } catch (const Fail& f) {
    return f.s;
  } catch (const std::bad_alloc&) {
    return XC_ERR_OOM;
  }
  return XC_OK;
}

xc_status xc_pool_destroy(xc_pool* pool) {
  delete pool;
  return XC_OK;
}

xc_status xc_pool_info(xc_pool* pool, int32_t* live_pages, int32_t* free_pages, int32_t* live_seqs) {
  if (!pool) return XC_ERR_INVALID_ARG;
  const PageBook& b = pool->p->book;
  if (live_pages) *live_pages = b.live_pages();
  if (free_pages) *free_pages = b.n_pages() - b.live_pages();
  if (live_seqs) *live_seqs = b.live_seqs();
  return XC_OK;
}

xc_status xc_seq_new(xc_pool* pool, int32_t* seq) {
  if (!pool || !seq) return XC_ERR_INVALID_ARG;
  if (pool->p->sticky) return XC_ERR_HIP;
  return status_of(pool->p->book.create(seq));
}

xc_status xc_seq_fork(xc_pool* pool, int32_t src, int32_t n, int32_t* seqs) {
  if (!pool || n < 0 || (n > 0 && !seqs)) return XC_ERR_INVALID_ARG;
  if (pool->p->sticky) return XC_ERR_HIP;
  try {
    return status_of(pool->p->book.fork(src, n, seqs));
  } catch (const std::bad_alloc&) {
    return XC_ERR_OOM;
  }
}

xc_status xc_seq_extend(xc_pool* pool, int32_t n, const int32_t* seqs, const int32_t* tokens) {
  if (!pool || n < 0 || (n > 0 && (!seqs || !tokens))) return XC_ERR_INVALID_ARG;
  Pool& p = *pool->p;
  return guarded(p, [&]() -> xc_status {
    if (capturing(p.st)) return XC_ERR_STATE;
    std::vector<PageCopy> copies;
    const PageStatus s = p.book.extend(n, seqs, tokens, &copies);
    if (s != PageStatus::ok) return status_of(s);
    committed([&] { copy_pages(p, copies); });
    return XC_OK;
  });
}

xc_status xc_seq_trim(xc_pool* pool, int32_t seq, int32_t front, int32_t back) {
  if (!pool) return XC_ERR_INVALID_ARG;
  if (pool->p->sticky) return XC_ERR_HIP;
  return status_of(pool->p->book.trim(seq, front, back));
}

xc_status xc_seq_free(xc_pool* pool, int32_t n, const int32_t* seqs) {
  if (!pool || n < 0 || (n > 0 && !seqs)) return XC_ERR_INVALID_ARG;
  if (pool->p->sticky) return XC_ERR_HIP;
  try {
    return status_of(pool->p->book.free(n, seqs));
  } catch (const std::bad_alloc&) {
    return XC_ERR_OOM;
  }
}

xc_status xc_pool_compact(xc_pool* pool, int32_t* moved) {
  if (!pool) return XC_ERR_INVALID_ARG;
  Pool& p = *pool->p;
  return guarded(p, [&]() -> xc_status {
    if (capturing(p.st)) return XC_ERR_STATE;
    std::vector<PageCopy> moves;
    p.book.compact(&moves);
    if (moved) *moved = (int32_t)moves.size();
    committed([&] { copy_pages(p, moves); });
    return XC_OK;
  });
}

xc_status xc_seq_pages(xc_pool* pool, int32_t seq, int32_t* first, int32_t* tokens, int32_t* pages, size_t cap,
                       size_t* n_pages) {
  if (!pool || !pool->p->book.valid(seq)) return XC_ERR_INVALID_ARG;
  const PageSeq& q = pool->p->book.seq(seq);
  if (first) *first = q.first;
  if (tokens) *tokens = q.tokens;
  if (n_pages) *n_pages = q.pages.size();
  if (pages)
    for (size_t i = 0; i < q.pages.size() && i < cap; ++i) pages[i] = q.pages[i];
  return XC_OK;
}

xc_status xc_seq_import(xc_pool* pool, int32_t seq, xc_handle* h) {
  if (!pool || !h || !pool->p->book.valid(seq)) return XC_ERR_INVALID_ARG;
  Pool& p = *pool->p;
  return guarded(p, [&]() -> xc_status {
    const HandleWindow w = handle_window(h);
    if (w.sticky) return XC_ERR_HIP;
    if (w.device != p.device || w.st != p.st || w.dtype != p.cfg.dtype || w.n_blocks != p.cfg.n_blocks ||
        w.heads != p.cfg.kv_heads || w.D != p.cfg.head_dim)
      return XC_ERR_INVALID_ARG;
    if (capturing(p.st)) return XC_ERR_STATE;
    if ((long long)w.chunks * w.tokens > kMaxPlaces) return XC_ERR_OOM;
    const int32_t n = w.chunks * w.tokens;
    std::vector<PageCopy> copies;
    const PageStatus s = p.book.extend(1, &seq, &n, &copies);
    if (s != PageStatus::ok) return status_of(s);
    committed([&] {
      copy_pages(p, copies);
      const PageSeq& q = p.book.seq(seq);
      const int shift = p.book.shift();
      int at = q.first + q.tokens - n;
      for (int slot : w.slots)
        for (int t = 0; t < w.tokens;) {
          ImportArgs a;
          const int page0 = at >> shift, place0 = at & (p.book.page() - 1);
          a.n_pages = std::min(kImportPages, (int)q.pages.size() - page0);
          std::copy(q.pages.begin() + page0, q.pages.begin() + page0 + a.n_pages, a.page);
          const int m = std::min(w.tokens - t, (a.n_pages << shift) - place0);
          XC_HIP(launch_import(a, w, slot, t, place0, m, p.block(0), p.block_elems(), p.st));
          t += m;
          at += m;
        }
    });
    return XC_OK;
  });
}

xc_status xc_batch_init(xc_pool* pool, xc_batch** out) {
  if (!pool || !out) return XC_ERR_INVALID_ARG;
  *out = new (std::nothrow) xc_batch;
  if (!*out) return XC_ERR_OOM;
  (*out)->p = pool->p;
  return XC_OK;
}

xc_status xc_batch_destroy(xc_batch* b) {
  if (!b) return XC_OK;
  if (capturing(b->p->st)) return XC_ERR_STATE;  // waiting would end the capture
  try {
    const DeviceScope scope(b->p->device);
    const OutsideCapture outside;
    if (b->dev || b->pieces || b->parts || b->evict || b->pinned) (void)hipStreamSynchronize(b->p->st);
    if (b->dev) (void)hipFree(b->dev);
    if (b->pieces) (void)hipFree(b->pieces);
    if (b->parts) (void)hipFree(b->parts);
    if (b->evict) (void)hipFree(b->evict);
    if (b->pinned) (void)hipHostFree(b->pinned);
    if (b->uploaded) (void)hipEventDestroy(b->uploaded);
  } catch (const Fail&) {
  }
  delete b;
  return XC_OK;
}

xc_status xc_batch_set(xc_batch* b, int32_t n, const int32_t* seqs, const int32_t* new_tokens) {
  if (!b || n < 0 || (n > 0 && (!seqs || !new_tokens))) return XC_ERR_INVALID_ARG;
  const xc_status s = guarded(*b->p, [&]() -> xc_status {
    if (!b->p->book.distinct(n, seqs)) return XC_ERR_INVALID_ARG;
    if (capturing(b->p->st)) return XC_ERR_STATE;
    const OutsideCapture outside;
    return set_batch(b, n, seqs, new_tokens);
  });
  if (s == XC_ERR_OOM || s == XC_ERR_HIP) b->set = false, b->rows = 0;  // wherever it failed
  return s;
}

xc_status xc_qk_norm_rope(xc_batch* b, int32_t block, const void* qkv, int64_t ld, const float* gq, const float* gk,
                          const int32_t* positions, int32_t n_axes, double theta, void* q_out, int64_t q_ld) {
  if (!b || !gq || !gk || (b->rows > 0 && (!qkv || !q_out))) return XC_ERR_INVALID_ARG;
  Pool& p = *b->p;
  const xc_pool_config& c = p.cfg;
  const long long width = (long long)(c.q_heads + 2 * c.kv_heads) * c.head_dim, q_width = (long long)c.q_heads * c.head_dim;
  if (block < 0 || block >= c.n_blocks || ld < width || q_ld < q_width || ld > kMaxStride || q_ld > kMaxStride ||
      ld * p.esz % 16 || q_ld * p.esz % 16 || !aligned16(qkv) || !aligned16(q_out))
    return XC_ERR_INVALID_ARG;
  if (positions && ((n_axes != 1 && n_axes != 3) || !std::isfinite(theta) || theta <= 1.0)) return XC_ERR_INVALID_ARG;
  return guarded(p, [&]() -> xc_status {
    if (!b->current()) return XC_ERR_STATE;
    const Rows in = rows_at(qkv, b->rows, ld, width, p.esz), to = rows_at(q_out, b->rows, q_ld, q_width, p.esz);
    if (overlap(in, to) || p.holds(qkv, in.extent) || p.holds(q_out, to.extent)) return XC_ERR_INVALID_ARG;
    // a page that another sequence reads too is not written
    for (int page : b->written)
      if (p.book.refs(page) > 1) return XC_ERR_STATE;
    if (b->rows == 0) return XC_OK;
    NormRopeArgs a{};
    a.qkv = qkv;
    a.ld = ld;
    a.gq = gq;
    a.gk = gk;
    a.positions = positions;
    a.q_out = q_out;
    a.q_ld = q_ld;
    a.place = b->place;
    a.rows = b->rows;
    a.q_heads = c.q_heads;
    a.buf = p.block(block);
    if (positions) {
      if (p.theta != theta || p.freqs.axes != n_axes) p.freqs = rope_freqs(c.head_dim, n_axes, theta), p.theta = theta;
      a.freqs = p.freqs;
    }
    XC_HIP(launch_norm_rope(c.dtype, a, p.st));
    return XC_OK;
  });
}

xc_status xc_branch_attention(xc_batch* b, int32_t block, const void* q, int64_t q_ld, float scale, void* out,
                              int64_t out_ld) {
  if (!b || (b->rows > 0 && (!q || !out))) return XC_ERR_INVALID_ARG;
  Pool& p = *b->p;
  const xc_pool_config& c = p.cfg;
  const long long width = (long long)c.q_heads * c.head_dim;
  if (block < 0 || block >= c.n_blocks || q_ld < width || out_ld < width || q_ld > kMaxStride || out_ld > kMaxStride ||
      q_ld * p.esz % 16 || out_ld * p.esz % 16 || !aligned16(q) || !aligned16(out))
    return XC_ERR_INVALID_ARG;
  const float log2_scale = (scale == 0.f ? 1.0f / std::sqrt((float)c.head_dim) : scale) * 1.4426950408889634f;
  if (!(scale >= 0.f) || !std::isnormal(log2_scale)) return XC_ERR_INVALID_ARG;
  return guarded(p, [&]() -> xc_status {
    if (!b->current() || b->chunk) return XC_ERR_STATE;
    const Rows in = rows_at(q, b->rows, q_ld, width, p.esz), to = rows_at(out, b->rows, out_ld, width, p.esz);
    if (overlap(in, to) || p.holds(out, to.extent)) return XC_ERR_INVALID_ARG;
    if (b->rows == 0) return XC_OK;
    AttnArgs a = b->attn;
    a.q = q;
    a.q_ld = q_ld;
    a.out = out;
    a.out_ld = out_ld;
    a.buf = p.block(block);
    a.scale = log2_scale;
    XC_HIP(launch_branch_attention(c.dtype, a, p.st));
    return XC_OK;
  });
}

}  // extern "C"
