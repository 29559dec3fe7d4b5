// Kernels of the branching cache besides its attention: page copies, the
// import of a model handle's window, the rows of a batch, and the per-head
// norms with the rotation that write new keys and values into pages.
//
// All are bound by HBM (or, with few rows, by latency): every one moves
// 16 bytes per lane and load, with several loads in flight per wave.
#include "xc_pool.h"

#include "xc_internal.h"

#include <math.h>

namespace xc {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}

// Sum over aligned runs of N lanes (8, 16 or 32), the same in each of them:
// every step adds the two halves of a run in either order.
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp_move<0xB1>(v);   // lane ^ 1
  v += dpp_move<0x4E>(v);   // lane ^ 2
  v += dpp_move<0x141>(v);  // the two quads of 8 lanes
  if (N >= 16) v += dpp_move<0x140>(v);  // the two halves of a row of 16
  if (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// What a call moves past this many bytes cannot stay in the 256 MB cache before
// memory until somebody reads it, and goes round it.  Measured both ways:
//   norms and rotation, 516 MB:  88 us round it,  99 us through it
//   norms and rotation,  60 MB:  14.5 us,         13.5 us
//   page copies, 369 MB:         75 us,           82 us
//   page copies,  10 MB:          5.9 us,          4.7 us
constexpr long long kBeyondCache = 256ll << 20;

// Rows [0, rows) of every head of page src to page dst, in keys or values of
// one block: a workgroup moves up to 16 KB, its loads issued together (8 a
// thread instead of 4: 119 us instead of 82 for 369 MB).  Bytes alone (both
// sides of a copy are whole 16-byte chunks).  ROUND: the loads pass the cache by.
constexpr int kCopyLoads = 4;
template <int N, bool ROUND>
__global__ __launch_bounds__(256) void page_copy_kernel(CopyArgs<N> a, char* keys, char* values, int kv_heads,
                                                        unsigned row_chunks, int page, long long block_bytes) {
  const PageCopy c = a.c[blockIdx.y];
  const unsigned head_chunks = page * row_chunks, seg = c.rows * row_chunks, total = kv_heads * seg;
  char* base = (blockIdx.z & 1 ? values : keys) + (blockIdx.z >> 1) * block_bytes;
  const u32x4* src = reinterpret_cast<const u32x4*>(base) + (long long)c.src * kv_heads * head_chunks;
  u32x4* dst = reinterpret_cast<u32x4*>(base) + (long long)c.dst * kv_heads * head_chunks;
  unsigned at[kCopyLoads];
  u32x4 v[kCopyLoads];
#pragma unroll
  for (int u = 0; u < kCopyLoads; ++u) {
    const unsigned i = (blockIdx.x * kCopyLoads + u) * 256 + threadIdx.x;
    const unsigned h = i / seg;
    at[u] = i < total ? h * head_chunks + (i - h * seg) : ~0u;
    if (at[u] != ~0u) v[u] = ROUND ? __builtin_nontemporal_load(src + at[u]) : src[at[u]];
  }
#pragma unroll
  for (int u = 0; u < kCopyLoads; ++u)
    if (at[u] != ~0u) dst[at[u]] = v[u];
}

// Tokens [0, n) of one chunk slot of a handle's cache (K [H][Lcap][D],
// V^T [H][D][Lcap], Lcap a multiple of 64) to places place0 .. of the listed
// pages.  A workgroup takes 64 tokens of one head of one block; V^T is read
// from the 16-byte boundary before its first token and turned through LDS.
// 2 chunks of 7020 tokens, 12 heads of 128, 2 blocks (345 MB read and written):
// 84 us, 177 with an element per load and store.
template <typename T>
__global__ __launch_bounds__(256) void import_kernel(ImportArgs a, const T* __restrict__ keys,
                                                     const T* __restrict__ values, long long Lcap, long long col0,
                                                     int place0, int n, T* __restrict__ pk, T* __restrict__ pv,
                                                     int shift, int D, long long block_elems) {
  constexpr int V = 16 / sizeof(T), COLS = 64 / V + 1, U = 5;
  typedef T vec __attribute__((ext_vector_type(V)));
  __shared__ __attribute__((aligned(16))) T tile[64 * (128 + V)];
  const int H = gridDim.y, h = blockIdx.y, b = blockIdx.z, t0 = blockIdx.x * 64, pitch = D + V, per_row = D / V;
  const int m = min(64, n - t0);
  const long long head = ((long long)b * H + h) * Lcap * D;
  auto dst = [&](int t) __attribute__((always_inline)) {
    const int at = place0 + t0 + t;
    return b * block_elems + ((((long long)a.page[at >> shift] * H + h) << shift) + (at & ((1 << shift) - 1))) * D;
  };
  const long long first = col0 + t0, base = first & ~(long long)(V - 1);
  const int skip = (int)(first - base);
  for (int i0 = threadIdx.x; i0 < D * COLS; i0 += 256 * U) {
    vec x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + 256 * u, d = i / COLS, c = i % COLS;
      if (i < D * COLS && c * V < skip + m)
        x[u] = *reinterpret_cast<const vec*>(values + head + d * Lcap + base + c * V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + 256 * u, d = i / COLS, c = i % COLS;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int t = c * V + e - skip;
        if (i < D * COLS && t >= 0 && t < m) tile[t * pitch + d] = x[u][e];
      }
    }
  }
  const vec* src = reinterpret_cast<const vec*>(keys + head + first * D);  // rows on end
  for (int i0 = threadIdx.x; i0 < m * per_row; i0 += 256 * U) {
    vec x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + 256 * u < m * per_row) x[u] = src[i0 + 256 * u];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + 256 * u, t = i / per_row;
      if (i < m * per_row) *reinterpret_cast<vec*>(pk + dst(t) + (i - t * per_row) * V) = x[u];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < m * per_row; i += 256) {
    const int t = i / per_row, c = (i - t * per_row) * V;
    *reinterpret_cast<vec*>(pv + dst(t) + c) = *reinterpret_cast<const vec*>(&tile[t * pitch + c]);
  }
}

__global__ __launch_bounds__(256) void batch_rows_kernel(const int* __restrict__ tables,
                                                         const BatchSeq* __restrict__ seqs, int n, int rows, int shift,
                                                         int* __restrict__ place, OwnSlots* __restrict__ own) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row >= rows) return;
  int lo = 0, hi = n;  // the last sequence with row0 <= row
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (seqs[mid].row0 <= row) lo = mid;
    else hi = mid;
  }
  const BatchSeq s = seqs[lo];
  const int at = s.at + row - s.row0;
  place[row] = (tables[s.table + (at >> shift)] << shift) + (at & ((1 << shift) - 1));
  own[row] = s.own;
}

// Per-head RMSNorm of q and k with gains, rotation, and k / v to their pages,
// one pass: x r g with r = 1 / sqrt(mean x^2 + 1e-6), then pair (2i, 2i + 1)
// turned by position * theta^(-2i / d_a).  One rounding, at the store.
//
// A lane holds 16 bytes of one head (D / E lanes a head), so both numbers of
// every pair are its own and the sum of squares stays within a row of lanes.
// A wave keeps to one row: its lanes meet the same dims in every head, so the
// angles are formed once, a pair per lane, and serve all heads (a lane that
// formed all the pairs it needs: 14.2 us instead of 12.9 for 9800 rows of
// (16 + 2 x 4) x 64).  Angles are turns (revolutions) in double - positions
// reach 2^31, where a float has lost the fraction - and only the fraction of a
// turn goes on to sincospi in float.
//
// ROUND: loads and stores pass the cache by.
template <typename T, int D, bool ROUND>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormRopeArgs a, int parts, int groups) {
  constexpr int E = 16 / sizeof(T), LPH = D / E, HPW = 64 / LPH, U = ROUND ? 5 : 4;
  typedef T vec __attribute__((ext_vector_type(E)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long w = (long long)blockIdx.x * 4 + wave;
  const int row = (int)(w / parts), part = (int)(w - (long long)row * parts);
  if (row >= a.rows) return;
  const int kv = a.buf.kv_heads, n_heads = a.q_heads + 2 * kv;
  const int sub = lane / LPH, d0 = (lane % LPH) * E;
  const int all = (n_heads + HPW - 1) / HPW;
  const int g0 = part * groups, g1 = min(g0 + groups, all);
  const T* src = reinterpret_cast<const T*>(a.qkv) + row * a.ld + d0;
  vec x[U];
  auto load = [&](int g) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int head = (g + u) * HPW + sub;
      const vec* p = reinterpret_cast<const vec*>(src + (long long)head * D);
      if (g + u < g1 && head < n_heads) x[u] = ROUND ? __builtin_nontemporal_load(p) : *p;
    }
  };
  load(g0);
  const int place = a.place[row];
  float gain[2][E], c[E / 2], s[E / 2];
#pragma unroll
  for (int i = 0; i < E; ++i) gain[0][i] = a.gq[d0 + i], gain[1][i] = a.gk[d0 + i];
#pragma unroll
  for (int i = 0; i < E / 2; ++i) c[i] = 1.f, s[i] = 0.f;
  if (a.positions != nullptr) {
    const int pair = lane % (D / 2);
    const int axis = pair < a.freqs.n0 ? 0 : pair < a.freqs.n0 + a.freqs.n1 ? 1 : 2;
    const double t = (double)a.positions[(long long)row * a.freqs.axes + axis] * a.freqs.turns[pair];
    float sv, cv;
    sincospif(2.f * (float)(t - rint(t)), &sv, &cv);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      c[i] = __shfl(cv, d0 / 2 + i, 64);
      s[i] = __shfl(sv, d0 / 2 + i, 64);
    }
  }
  const int shift = a.buf.shift;
  const long long page = place >> shift, r = place & ((1 << shift) - 1);
  T* kd = reinterpret_cast<T*>(a.buf.keys);
  T* vd = reinterpret_cast<T*>(a.buf.values);
  T* qd = reinterpret_cast<T*>(a.q_out) + row * a.q_ld;
  for (int g = g0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int head = (g + u) * HPW + sub;
      if (g + u >= g1) break;
      const bool is_q = head < a.q_heads, is_v = head >= a.q_heads + kv;
      float f[E], ss = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] = head < n_heads ? (float)x[u][i] : 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) ss += f[i] * f[i];
      ss = lanes_sum<LPH>(ss);
      const float rn = 1.0f / sqrtf(ss * (1.0f / D) + 1e-6f);
      vec y = x[u];
      if (!is_v) {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] *= rn * (is_q ? gain[0][i] : gain[1][i]);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          y[2 * i] = (T)(f[2 * i] * c[i] - f[2 * i + 1] * s[i]);
          y[2 * i + 1] = (T)(f[2 * i] * s[i] + f[2 * i + 1] * c[i]);
        }
      }
      T* dst = is_q ? qd + (long long)head * D
                    : (is_v ? vd : kd) +
                          (((page * kv + head - a.q_heads - (is_v ? kv : 0)) << shift) + r) * D;
      if (head < n_heads) {
        if (ROUND) __builtin_nontemporal_store(y, reinterpret_cast<vec*>(dst + d0));
        else *reinterpret_cast<vec*>(dst + d0) = y;
      }
    }
    g += U;
    if (g >= g1) break;
    load(g);
  }
}

}  // namespace

namespace {
template <int N>
void page_copies(const PageCopy* copies, int n, const PageBuf& whole, int esz, int n_blocks, long long block_bytes,
                 hipStream_t st) {
  const int page = 1 << whole.shift, row_chunks = whole.D * esz / 16;
  CopyArgs<N> a;
  int most = 0;
  long long rows = 0;
  for (int i = 0; i < n; ++i) {
    a.c[i] = copies[i];
    rows += copies[i].rows;
    most = copies[i].rows > most ? copies[i].rows : most;
  }
  const long long chunks = (long long)whole.kv_heads * most * row_chunks;
  const dim3 grid((unsigned)((chunks + 256 * kCopyLoads - 1) / (256 * kCopyLoads)), n, 2 * n_blocks);
  const bool round = 2 * rows * whole.kv_heads * row_chunks * 16 * 2 * n_blocks > kBeyondCache;  // read and written
#define XC_COPY(ROUND)                                                                                             \
  page_copy_kernel<N, ROUND><<<grid, 256, 0, st>>>(a, (char*)whole.keys, (char*)whole.values, whole.kv_heads,      \
                                                   row_chunks, page, block_bytes)
  if (round) XC_COPY(true);
  else XC_COPY(false);
#undef XC_COPY
}
}  // namespace

hipError_t launch_page_copies(const PageCopy* copies, int n, const PageBuf& whole, int esz, int n_blocks,
                              long long block_bytes, hipStream_t st) {
  if (n <= kCopyBatchFew) page_copies<kCopyBatchFew>(copies, n, whole, esz, n_blocks, block_bytes, st);
  else page_copies<kCopyBatch>(copies, n, whole, esz, n_blocks, block_bytes, st);
  return hipGetLastError();
}

hipError_t launch_import(const ImportArgs& a, const HandleWindow& w, int slot, int chunk_token, int place0, int n_tokens,
                         const PageBuf& whole, long long block_elems, hipStream_t st) {
  const dim3 grid((n_tokens + 63) / 64, w.heads, w.n_blocks);
  const long long col0 = (long long)slot * w.tokens + chunk_token;
  if (w.dtype == 1)
    import_kernel<bf16><<<grid, 256, 0, st>>>(a, (const bf16*)w.keys, (const bf16*)w.values, w.Lcap, col0, place0,
                                              n_tokens, (bf16*)whole.keys, (bf16*)whole.values, whole.shift, w.D,
                                              block_elems);
  else
    import_kernel<float><<<grid, 256, 0, st>>>(a, (const float*)w.keys, (const float*)w.values, w.Lcap, col0, place0,
                                               n_tokens, (float*)whole.keys, (float*)whole.values, whole.shift, w.D,
                                               block_elems);
  return hipGetLastError();
}

hipError_t launch_batch_rows(const int* tables, const BatchSeq* seqs, int n, int rows, int shift, int* place,
                             OwnSlots* own, hipStream_t st) {
  batch_rows_kernel<<<(rows + 255) / 256, 256, 0, st>>>(tables, seqs, n, rows, shift, place, own);
  return hipGetLastError();
}

hipError_t launch_norm_rope(int dtype, const NormRopeArgs& a, hipStream_t st) {
  const int per_wave = 64 / (a.buf.D * (dtype == 1 ? 2 : 4) / 16);
  const int all = (a.q_heads + 2 * a.buf.kv_heads + per_wave - 1) / per_wave;
  // few rows: their heads are dealt to several waves
  int groups = all;
  while (groups > 1 && (long long)a.rows * ((all + groups - 1) / groups) < 4096) groups = (groups + 1) / 2;
  const int parts = (all + groups - 1) / groups;
  const unsigned grid = (unsigned)(((long long)a.rows * parts + 3) / 4);
  const bool round = 2ll * a.rows * (a.q_heads + 2 * a.buf.kv_heads) * a.buf.D * (dtype == 1 ? 2 : 4) > kBeyondCache;
#define XC_NORM(T, DD)                                                                 \
  do {                                                                                 \
    if (round) norm_rope_kernel<T, DD, true><<<grid, 256, 0, st>>>(a, parts, groups);  \
    else norm_rope_kernel<T, DD, false><<<grid, 256, 0, st>>>(a, parts, groups);       \
  } while (0)
  if (dtype == 1) {
    if (a.buf.D == 128) XC_NORM(bf16, 128);
    else XC_NORM(bf16, 64);
  } else {
    if (a.buf.D == 128) XC_NORM(float, 128);
    else if (a.buf.D == 64) XC_NORM(float, 64);
    else XC_NORM(float, 32);
  }
#undef XC_NORM
  return hipGetLastError();
}

}  // namespace xc
