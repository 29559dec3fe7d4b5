// State of the branching cache's host side (xc_pool, xc_batch in
// include/xcache.h) and what its entry points have in common: failures, the
// pool's device, capture, buffers that grow, rows that overlap.
#pragma once

#include <hip/hip_runtime.h>

#include <cstring>
#include <memory>
#include <new>
#include <vector>

#include "xc_chunk.h"
#include "xc_internal.h"
#include "xc_pool.h"
#include "xcache.h"

namespace xc {

// places (page * page tokens + row) are 32-bit numbers with room for a tile
constexpr long long kMaxPlaces = 1ll << 30;
constexpr int kMaxRows = 1 << 24;
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

inline xc_status status_of(PageStatus s) {
  return s == PageStatus::ok ? XC_OK : s == PageStatus::full ? XC_ERR_OOM : XC_ERR_INVALID_ARG;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
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
inline bool capturing(hipStream_t st) {
  hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(st, &s) != hipSuccess) {
    (void)hipGetLastError();
    return true;
  }
  return s != hipStreamCaptureStatusNone;
}

}  // namespace xc

struct xc_pool {
  std::shared_ptr<xc::Pool> p;
};

struct xc_batch {
  std::shared_ptr<xc::Pool> p;
  // what xc_batch_set or xc_chunk_set left
  bool set = false, chunk = false;  // chunk: rows under a mask
  std::vector<int> seqs;
  std::vector<uint64_t> versions;
  std::vector<int> written;  // pages that hold rows of the batch
  xc::AttnArgs attn{};       // the plan's part of the arguments
  const int* place = nullptr;
  int rows = 0;
  xc::WeightArgs weights{};  // of a chunk batch
  // buffers
  char* dev = nullptr;
  size_t dev_bytes = 0;
  char* pieces = nullptr;
  size_t piece_bytes = 0;
  char* parts = nullptr;  // partial sums of weights; parts_need: of the rows that are set
  size_t parts_bytes = 0, parts_need = 0;
  char* evict = nullptr;  // an eviction's tables and choices
  size_t evict_bytes = 0;
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

namespace xc {

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

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// A caller's [rows][ld], `width` elements of each row in use; all in bytes.
struct Rows {
  uintptr_t at;
  size_t pitch, width, extent;  // extent: to the end of the last row
};
inline Rows rows_at(const void* p, long long rows, long long ld, long long width, int esz) {
  return {reinterpret_cast<uintptr_t>(p), (size_t)ld * esz, (size_t)width * esz,
          rows > 0 ? (size_t)((rows - 1) * ld + width) * esz : 0};
}
// Rows of one stride may lie beside each other in a buffer; others are told apart by where they begin and end.
inline bool overlap(const Rows& a, const Rows& b) {
  if (a.at >= b.at + b.extent || b.at >= a.at + a.extent) return false;
  if (a.pitch != b.pitch) return true;
  const size_t from = b.at >= a.at ? (b.at - a.at) % a.pitch : (a.pitch - (a.at - b.at) % a.pitch) % a.pitch;
  return from < a.width || from + b.width > a.pitch;
}

// Device memory of at least `need` bytes at buf, its contents lost; false: there is none.  Work before may still use the
// smaller buffer, and is waited for.
inline bool enlarge(Pool& p, char*& buf, size_t& have, size_t need, size_t reserve) {
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

// Room for `need` bytes at dev, of which `up` are uploaded; false: there is none.
inline bool staging(xc_batch* b, char*& dev, size_t& have, size_t need, size_t up) {
  if (!enlarge(*b->p, dev, have, need, need / 2)) return false;
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
  return true;
}
// ... and its contents, the staging memory written from `at` on
template <typename T>
void put(xc_batch* b, size_t at, const std::vector<T>& v) {
  if (!v.empty()) std::memcpy(b->pinned + at, v.data(), v.size() * sizeof(T));
}
inline void upload(xc_batch* b, char* dev, size_t up) {
  XC_HIP(hipMemcpyAsync(dev, b->pinned, up, hipMemcpyHostToDevice, b->p->st));
  XC_HIP(hipEventRecord(b->uploaded, b->p->st));
  b->upload_pending = true;
}

// The sequences of a batch that have rows.
struct BatchRows {
  std::vector<PlanSeq> seqs;
  std::vector<int> number;  // of the batch's sequences
  std::vector<int> tables, written, first_row;
  std::vector<uint64_t> versions;  // of all its sequences
  int rows = 0;
  int shared_end = 0;  // the place up to which their pages are the same ones, whole pages
};
inline xc_status batch_rows(const Pool& p, int32_t n, const int32_t* seqs, const int32_t* new_tokens, BatchRows* out) {
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
  out->shared_end = with_rows < 2 ? 0 : (int)(shared << shift);
  out->rows = (int)rows;
  out->versions.resize(n);
  int row0 = 0;
  for (int i = 0; i < n; ++i) {
    const PageSeq& q = book.seq(seqs[i]);
    out->versions[i] = q.version;
    if (new_tokens[i] == 0) continue;
    const int at = q.first + q.tokens - new_tokens[i];
    out->seqs.push_back({new_tokens[i], q.first, q.tokens, (int)out->tables.size()});
    out->number.push_back(i);
    out->first_row.push_back(row0);
    out->tables.insert(out->tables.end(), q.pages.begin(), q.pages.end());
    out->written.insert(out->written.end(), q.pages.begin() + (at >> shift), q.pages.end());
    row0 += new_tokens[i];
  }
  return out->tables.size() > (size_t)kMaxPlaces ? XC_ERR_UNSUPPORTED : XC_OK;
}

}  // namespace xc
