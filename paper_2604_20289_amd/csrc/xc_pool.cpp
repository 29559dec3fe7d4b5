// Host side of the branching cache (xc_pool, xc_batch in include/xcache.h):
// argument validation, page tables, the plan of a batch and the launches.
//
// Device state of a batch: the page tables of its sequences, the attention's
// units and, per row, the place its token has in the pages and the slots of
// its pieces; and the pieces themselves.  Tables go up from pinned memory on
// the pool's stream.  A buffer that became too small goes once the work before
// is done (a graph captured before is not replayed after a new xc_batch_set).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <vector>

#include "xc_internal.h"
#include "xc_pool.h"
#include "xcache.h"

using namespace xc;

namespace {

// places (page * page tokens + row) are 32-bit numbers with room for a tile
constexpr long long kMaxPlaces = 1ll << 30;
constexpr int kMaxRows = 1 << 24;
constexpr int kMaxHeads = 1024;
constexpr long long kMaxStride = 1ll << 36;  // a row stride; keeps extents in 64 bits

struct Fail {
  xc_status s;
};

#define XC_HIP(call)                                                              \
  do {                                                                            \
    const hipError_t e_ = (call);                                                 \
    if (e_ != hipSuccess) {                                                       \
      (void)hipGetLastError();                                                    \
      throw Fail{e_ == hipErrorOutOfMemory ? XC_ERR_OOM : XC_ERR_HIP};            \
    }                                                                             \
  } while (0)

// The pool's device for the length of a call.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    XC_HIP(hipGetDevice(&before_));
    if (before_ != device) {
      XC_HIP(hipSetDevice(device));
      changed_ = true;
    }
  }
  ~DeviceScope() {
    if (changed_) (void)hipSetDevice(before_);
  }

 private:
  int before_ = 0;
  bool changed_ = false;
};

// Allocations of a batch have nothing to do with a capture of some other stream, whose mode may forbid them to all.
class OutsideCapture {
 public:
  OutsideCapture() { XC_HIP(hipThreadExchangeStreamCaptureMode(&mode_)); }
  ~OutsideCapture() { (void)hipThreadExchangeStreamCaptureMode(&mode_); }

 private:
  hipStreamCaptureMode mode_ = hipStreamCaptureModeRelaxed;
};

xc_status status_of(PageStatus s) {
  return s == PageStatus::ok ? XC_OK : s == PageStatus::full ? XC_ERR_OOM : XC_ERR_INVALID_ARG;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + bn && y < x + an;
}

struct Pool {
  Pool(const xc_pool_config& c, int shift) : cfg(c), book(c.n_pages, shift, c.max_seqs) {}
  xc_pool_config cfg;
  PageBook book;
  char *keys = nullptr, *values = nullptr;
  hipStream_t st = nullptr;
  int device = 0, cus = 256, esz = 4;
  bool sticky = false;
  RopeFreqs freqs{};     // of (theta, axes): the same in every call of a model
  double theta = 0.0;

  long long block_elems() const {
    return ((long long)cfg.n_pages << book.shift()) * cfg.kv_heads * cfg.head_dim;
  }
  // whether bytes lie in the page buffers
  bool holds(const void* x, size_t n) const {
    const size_t bytes = (size_t)block_elems() * cfg.n_blocks * esz;
    return n > 0 && (overlap(x, n, keys, bytes) || overlap(x, n, values, bytes));
  }
  PageBuf block(int b) const {
    const long long o = b * block_elems() * esz;
    return {keys + o, values + o, book.shift(), cfg.kv_heads, cfg.head_dim};
  }
};

// Tables change on the host while the call is made: inside a capture the
// replayed work and they would part.
bool capturing(hipStream_t st) {
  hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(st, &s) != hipSuccess) {
    (void)hipGetLastError();
    return true;
  }
  return s != hipStreamCaptureStatusNone;
}

void copy_pages(Pool& p, const std::vector<PageCopy>& copies) {
  for (size_t i = 0; i < copies.size(); i += kCopyBatch)
    XC_HIP(launch_page_copies(copies.data() + i, (int)std::min<size_t>(kCopyBatch, copies.size() - i), p.block(0), p.esz,
                              p.cfg.n_blocks, p.block_elems() * p.esz, p.st));
}

}  // namespace

struct xc_pool {
  std::shared_ptr<Pool> p;
};

struct xc_batch {
  std::shared_ptr<Pool> p;
  // what xc_batch_set left
  bool set = false;
  std::vector<int> seqs;
  std::vector<uint64_t> versions;
  std::vector<int> written;  // pages that hold rows of the batch
  AttnArgs attn{};           // the plan's part of the arguments
  const int* place = nullptr;
  int rows = 0;
  // buffers
  char* dev = nullptr;
  size_t dev_bytes = 0;
  char* pieces = nullptr;
  size_t piece_bytes = 0;
  char* pinned = nullptr;
  size_t pinned_bytes = 0;
  hipEvent_t uploaded = nullptr;
  bool upload_pending = false;

  // the tables are still those of its sequences
  bool current() const {
    if (!set) return false;
    for (size_t i = 0; i < seqs.size(); ++i)
      if (!p->book.valid(seqs[i]) || p->book.seq(seqs[i]).version != versions[i]) return false;
    return true;
  }
};

namespace {

// Runs f with the pool's device current; failures of HIP stick to the pool.
template <typename F>
xc_status guarded(Pool& p, F&& f) {
  if (p.sticky) return XC_ERR_HIP;
  try {
    const DeviceScope scope(p.device);
    return f();
  } catch (const Fail& e) {
    if (e.s == XC_ERR_HIP) p.sticky = true;
    return e.s;
  } catch (const std::bad_alloc&) {
    return XC_ERR_OOM;
  }
}

// ... of a call that changes tables before it launches: a launch that fails
// leaves tables and pages apart, whatever the reason
template <typename F>
void committed(F&& f) {
  try {
    f();
  } catch (...) {
    throw Fail{XC_ERR_HIP};
  }
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// A caller's [rows][ld], `width` elements of each row in use; all in bytes.
struct Rows {
  uintptr_t at;
  size_t pitch, width, extent;  // extent: to the end of the last row
};
Rows rows_at(const void* p, long long rows, long long ld, long long width, int esz) {
  return {reinterpret_cast<uintptr_t>(p), (size_t)ld * esz, (size_t)width * esz,
          rows > 0 ? (size_t)((rows - 1) * ld + width) * esz : 0};
}
// Rows of one stride may lie beside each other in a buffer; others are told apart by where they begin and end.
bool overlap(const Rows& a, const Rows& b) {
  if (a.at >= b.at + b.extent || b.at >= a.at + a.extent) return false;
  if (a.pitch != b.pitch) return true;
  const size_t from = b.at >= a.at ? (b.at - a.at) % a.pitch : (a.pitch - (a.at - b.at) % a.pitch) % a.pitch;
  return from < a.width || from + b.width > a.pitch;
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

// Device memory of at least `need` bytes at buf, its contents lost; false: there is none.  Work before may still use the
// smaller buffer, and is waited for.
bool enlarge(Pool& p, char*& buf, size_t& have, size_t need, size_t reserve) {
  if (need <= have) return true;
  if (buf) {
    XC_HIP(hipStreamSynchronize(p.st));
    char* old = buf;
    buf = nullptr;
    have = 0;
    XC_HIP(hipFree(old));
  }
  void* d = nullptr;
  const hipError_t e = hipMalloc(&d, need + reserve);
  if (e == hipErrorOutOfMemory) return (void)hipGetLastError(), false;
  XC_HIP(e);
  buf = (char*)d;
  have = need + reserve;
  return true;
}

xc_status set_batch(xc_batch* b, int32_t n, const int32_t* seqs, const int32_t* new_tokens) {
  Pool& p = *b->p;
  const PageBook& book = p.book;
  const int shift = book.shift();
  long long rows = 0;
  for (int i = 0; i < n; ++i) {
    if (new_tokens[i] < 0 || new_tokens[i] > book.seq(seqs[i]).tokens) return XC_ERR_INVALID_ARG;
    rows += new_tokens[i];
  }
  if (rows > kMaxRows) return XC_ERR_UNSUPPORTED;

  // whole pages that every sequence with rows begins with
  const PageSeq* head = nullptr;
  size_t shared = 0, with_rows = 0;
  for (int i = 0; i < n; ++i) {
    if (new_tokens[i] == 0) continue;
    const PageSeq& q = book.seq(seqs[i]);
    const size_t whole = (size_t)(((long long)q.first + q.tokens) >> shift);
    if (with_rows++ == 0) {
      head = &q;
      shared = whole;
      continue;
    }
    if (q.first != head->first) shared = 0;
    shared = std::min(shared, whole);
    size_t same = 0;
    while (same < shared && q.pages[same] == head->pages[same]) ++same;
    shared = same;
  }
  if (with_rows < 2) shared = 0;

  std::vector<PlanSeq> plan_seqs;
  std::vector<BatchSeq> batch_seqs;
  std::vector<int> tables, written, first_row;
  std::vector<uint64_t> versions(n);
  int row0 = 0;
  for (int i = 0; i < n; ++i) {
    const PageSeq& q = book.seq(seqs[i]);
    versions[i] = q.version;
    if (new_tokens[i] == 0) continue;
    const int at = q.first + q.tokens - new_tokens[i];
    plan_seqs.push_back({new_tokens[i], q.first, q.tokens, (int)tables.size()});
    first_row.push_back(row0);
    tables.insert(tables.end(), q.pages.begin(), q.pages.end());
    written.insert(written.end(), q.pages.begin() + (at >> shift), q.pages.end());
    row0 += new_tokens[i];
  }
  if (tables.size() > (size_t)kMaxPlaces) return XC_ERR_UNSUPPORTED;
  const int group = p.cfg.q_heads / p.cfg.kv_heads;
  const PlanShape shape{group, p.cfg.kv_heads, p.cfg.head_dim, p.esz, p.cus};
  AttnPlan plan = plan_attention(plan_seqs, (int)(shared << shift), shape);
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
    plan = plan_attention(plan_seqs, (int)(shared << shift), shape, 0);  // no memory: without pieces
    if (!launches()) return XC_ERR_OOM;
  }
  for (const PlanPart& part : plan.parts) {
    const PlanSeq& q = plan_seqs[part.seq];
    const int at = q.first + q.tokens - q.rows + (part.tok0 - first_row[part.seq]);
    batch_seqs.push_back({part.tok0, at, q.table, part.own});
  }

  // uploaded: tables, sequences, units; written on the device: places, own slots
  const size_t o_seqs = align256(tables.size() * sizeof(int));
  const size_t o_units = o_seqs + align256(batch_seqs.size() * sizeof(BatchSeq));
  const size_t up = o_units + align256(plan.units.size() * sizeof(AttnUnit));
  const size_t o_own = up + align256(rows * sizeof(int));
  const size_t need = o_own + align256(rows * sizeof(OwnSlots));
  std::vector<int> seq_copy(seqs, seqs + n);

  if (!enlarge(p, b->dev, b->dev_bytes, need, need / 2)) return XC_ERR_OOM;
  if (b->upload_pending) {  // the staging memory is being read
    XC_HIP(hipEventSynchronize(b->uploaded));
    b->upload_pending = false;
  }
  if (up > b->pinned_bytes) {
    void* d = nullptr;
    XC_HIP(hipHostMalloc(&d, up + up / 2, hipHostMallocDefault));
    if (b->pinned) (void)hipHostFree(b->pinned);
    b->pinned = (char*)d;
    b->pinned_bytes = up + up / 2;
  }
  if (!b->uploaded) XC_HIP(hipEventCreateWithFlags(&b->uploaded, hipEventDisableTiming));

  if (rows > 0) {
    std::memcpy(b->pinned, tables.data(), tables.size() * sizeof(int));
    std::memcpy(b->pinned + o_seqs, batch_seqs.data(), batch_seqs.size() * sizeof(BatchSeq));
    std::memcpy(b->pinned + o_units, plan.units.data(), plan.units.size() * sizeof(AttnUnit));
    XC_HIP(hipMemcpyAsync(b->dev, b->pinned, up, hipMemcpyHostToDevice, p.st));
    XC_HIP(hipEventRecord(b->uploaded, p.st));
    b->upload_pending = true;
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
  b->versions.swap(versions);
  b->written.swap(written);
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
    if (b->dev || b->pieces || b->pinned) (void)hipStreamSynchronize(b->p->st);
    if (b->dev) (void)hipFree(b->dev);
    if (b->pieces) (void)hipFree(b->pieces);
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
    if (!b->current()) return XC_ERR_STATE;
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
