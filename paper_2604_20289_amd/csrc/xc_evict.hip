// Evictions: which tokens a sequence keeps, and their keys and values moved
// to its first places.
#include "xc_chunk.h"

#include "xc_internal.h"

#include <math.h>

namespace xc {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Order of the weights as whole numbers: NaN below everything, -0 as +0.
__device__ __forceinline__ unsigned order_of(float w) {
  if (w != w) return 0u;
  const unsigned b = __float_as_uint(w + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sum of v over the lanes up to this one: within rows of 16, then the rows before.
__device__ __forceinline__ int lanes_up_to(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // the lane 1, 2, 4, 8 before
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // the last lane of row 0 to row 1, of 2 to 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // of row 1 to rows 2 and 3
  return v;
}
// Numbers of the waves before this one (totals, in LDS): their sum; all: of all waves.
template <int WAVES>
__device__ __forceinline__ int waves_before(const int* totals, int lane, int wave, int& all) {
  const int up = lanes_up_to(lane < WAVES ? totals[lane] : 0);
  all = __builtin_amdgcn_readlane(up, WAVES - 1);
  return wave == 0 ? 0 : __builtin_amdgcn_readlane(up, wave - 1);
}

// Which tokens a sequence keeps: the m-th largest weight of those that are
// neither among the first nor the last, by a search over the digits of its
// order (11, 11, 10 bits, a histogram each, until all of a digit's are wanted),
// then one pass in order that ranks
// and lists the kept ones and moves their weights.  A workgroup a sequence: its
// time is latency, of LDS and of barriers, 16 waves' or, for few tokens, 4's.
// Orders stay in registers where a thread has room for its own.
constexpr int kBins = 2048, kSelectFew = 4096;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a, int shift) {
  constexpr int WAVES = THREADS / 64, HELD = 24, ITEMS = 8, PER = kBins / THREADS;
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const EvictSeq s = a.seqs[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int* kept = a.kept ? a.kept + s.number * a.kept_ld : nullptr;
  if (s.keep < 0) {
    for (int t = tid; t < s.tokens; t += THREADS) kept[t] = t;
    return;
  }
  __shared__ __attribute__((aligned(16))) int hist[kBins][4];  // a copy for every fourth lane
  __shared__ int totals[2][WAVES];
  __shared__ int found[3];
  float* w = a.weights + s.number * a.ld;
  const int lo = a.sinks, hi = s.tokens - a.recent;
  int want = s.keep - a.sinks - a.recent;  // of them
  const bool any = want > 0, held = hi - lo <= HELD * THREADS;
  unsigned prefix = 0;                     // the digits found so far
  int below = 32;                          // the bits behind them
  unsigned order[HELD];
  if (any && held) {
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      const int t = lo + u * THREADS + tid;
      if (u * THREADS < hi - lo) order[u] = order_of(w[t < hi ? t : lo]);
    }
  }
  for (int pass = 0; pass < 3 && any; ++pass) {
    const int bits = pass == 2 ? 10 : 11, low = below - bits;
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<i32x4*>(hist[i * THREADS + tid]) = i32x4{0, 0, 0, 0};
    __syncthreads();
    auto count = [&](unsigned o, bool is) __attribute__((always_inline)) {
      if (is && (pass == 0 || o >> below == prefix)) atomicAdd(&hist[o >> low & ((1 << bits) - 1)][lane & 3], 1);
    };
    if (held) {
#pragma unroll
      for (int u = 0; u < HELD; ++u)
        if (u * THREADS < hi - lo) count(order[u], lo + u * THREADS + tid < hi);
    } else {
      for (int t0 = lo; t0 < hi; t0 += THREADS * ITEMS) {
        float x[ITEMS];
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
          const int t = t0 + u * THREADS + tid;
          x[u] = w[t < hi ? t : lo];
        }
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) count(order_of(x[u]), t0 + u * THREADS + tid < hi);
      }
    }
    __syncthreads();
    // bins from the top (those past a shorter digit's are empty): thread i has PER of them from number i * PER on
    int n[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const i32x4 c = *reinterpret_cast<const i32x4*>(hist[kBins - 1 - (tid * PER + k)]);
      n[k] = (c[0] + c[1]) + (c[2] + c[3]);
      sum += n[k];
    }
    const int up = lanes_up_to(sum);
    if (lane == 63) totals[0][wave] = up;
    __syncthreads();
    int all;
    int above = waves_before<WAVES>(totals[0], lane, wave, all) + up - sum;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if (above < want && above + n[k] >= want) found[0] = kBins - 1 - (tid * PER + k), found[1] = want - above, found[2] = n[k];
      above += n[k];
    }
    __syncthreads();
    prefix = prefix << bits | (unsigned)found[0];
    want = found[1];
    below = low;
    if (found[2] == want) break;
  }
  const int ties = want;  // of those as heavy as the lightest kept one, the first so many

  int tie0 = 0, kept0 = 0;  // before the tokens at hand
  for (int t0 = 0; t0 < s.tokens; t0 += THREADS * ITEMS) {
    float x[ITEMS];
    unsigned long long tie[ITEMS], sel[ITEMS];
    const int at = t0 + wave * 64 * ITEMS + lane;
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) x[u] = at + u * 64 < s.tokens ? w[at + u * 64] : 0.f;
    int n = 0;
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
      const int t = at + u * 64;
      tie[u] = __builtin_amdgcn_ballot_w64(any && t >= lo && t < hi && order_of(x[u]) >> below == prefix);
      n += __popcll(tie[u]);
    }
    if (lane == 0) totals[0][wave] = n;
    __syncthreads();
    int all;
    int rank = tie0 + waves_before<WAVES>(totals[0], lane, wave, all);
    tie0 += all;
    n = 0;
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
      const int t = at + u * 64, mine = rank + __popcll(tie[u] & ((1ull << lane) - 1));
      const bool is_tie = tie[u] >> lane & 1, mid = t >= lo && t < hi;
      sel[u] = __builtin_amdgcn_ballot_w64(t < s.tokens &&
                                           (!mid || (any && (is_tie ? mine < ties : order_of(x[u]) >> below > prefix))));
      rank += __popcll(tie[u]);
      n += __popcll(sel[u]);
    }
    if (lane == 0) totals[1][wave] = n;
    __syncthreads();
    int pos = kept0 + waves_before<WAVES>(totals[1], lane, wave, all);
    kept0 += all;
    // a kept token goes to its own place or a lower one, and all of this turn have been read
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
      const int t = at + u * 64, j = pos + __popcll(sel[u] & ((1ull << lane) - 1));
      if (sel[u] >> lane & 1) {
        const int place = s.first + t;
        a.src[s.at + j] = (a.tables[s.from + (place >> shift)] << shift) + (place & ((1 << shift) - 1));
        if (kept) kept[j] = t;
        w[j] = x[u];
      }
      pos += __popcll(sel[u]);
    }
    __syncthreads();
  }
  for (int t = s.keep + tid; t < s.tokens; t += THREADS) w[t] = 0.f;
}

// Kept tokens to their places, in keys or values of one head of one block, of
// each row one of `parts`.  One workgroup has them all, in order: a token's new
// place is its old one or a lower one, so what is loaded ahead has not been
// written over, and what is written over has been loaded: by every thread,
// before the barrier.  While a turn's rows are written, the next one's are on
// their way, and the places of the one after.  Bound by HBM: 12 sequences, 20
// blocks, 12 heads of 128 (2.3 GB) 357 us, 6.4 TB/s.
template <int LPR>
__global__ __launch_bounds__(512) void evict_move_kernel(EvictArgs a, char* keys, char* values, int shift, int kv, int parts,
                                                         long long block_bytes) {
  constexpr int ROWS = 512 / LPR, U = 4;  // 16-byte chunks of a row's part; rows of a turn: ROWS * U
  const EvictSeq s = a.seqs[blockIdx.z];
  if (s.keep <= 0) return;
  const int h = blockIdx.y / parts, c = blockIdx.y % parts * LPR + threadIdx.x % LPR, in_page = (1 << shift) - 1;
  u32x4* base = reinterpret_cast<u32x4*>((blockIdx.x & 1 ? values : keys) + (blockIdx.x >> 1) * block_bytes);
  auto at_of = [&](int place) __attribute__((always_inline)) {
    return ((((long long)(place >> shift) * kv + h) << shift) + (place & in_page)) * (LPR * parts) + c;
  };
  struct Turn {
    int from[U], to[U];
    u32x4 x[U];
  };
  auto places = [&](Turn& t, int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = min(j0 + u * ROWS + (int)threadIdx.x / LPR, s.keep - 1), place = s.first + j;
      t.from[u] = a.src[s.at + j];
      t.to[u] = (a.tables[s.to + (place >> shift)] << shift) + (place & in_page);
    }
  };
  auto load = [&](Turn& t) __attribute__((always_inline)) {
    // (a row that stays is not read: always the buffer's first one in its place, so that waits can count the loads)
#pragma unroll
    for (int u = 0; u < U; ++u) t.x[u] = base[t.from[u] != t.to[u] ? at_of(t.from[u]) : c];
  };
  // past the last row it is written again, by several threads alike
  auto store = [&](const Turn& t) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" ::"v"(t.x[u]));
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (t.from[u] != t.to[u]) base[at_of(t.to[u])] = t.x[u];
  };
  // tokens in pages before the last first one's stay
  const int sink_page = (s.first + min(a.sinks, s.keep)) >> shift << shift, j0 = max(0, sink_page - s.first);
  Turn t[2];
  places(t[0], j0);
  load(t[0]);
  places(t[1], j0 + ROWS * U);
  for (int j = j0; j < s.keep; j += 2 * ROWS * U) {
    load(t[1]);
    store(t[0]);
    places(t[0], j + 2 * ROWS * U);
    if (j + ROWS * U >= s.keep) break;
    load(t[0]);
    store(t[1]);
    places(t[1], j + 3 * ROWS * U);
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, const PageBuf& whole, int esz, int n_blocks, long long block_bytes, int most_tokens,
                        int most, hipStream_t st) {
  if (most_tokens <= kSelectFew) evict_select_kernel<256><<<a.n, 256, 0, st>>>(a, whole.shift);
  else evict_select_kernel<1024><<<a.n, 1024, 0, st>>>(a, whole.shift);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || most <= 0) return e;
  // A head's rows go through one workgroup, so few heads have few workgroups: parts of 128 bytes for fewer than four to a
  // CU, of 64 (half a line) for fewer than 192.  Measured, 21060 tokens back to 14040, 12 heads of 128 (rows of 256 bytes):
  // 2 blocks 154 us whole, 104 in halves, 89 in quarters; 4 blocks 172, 121, 131; 14 blocks 341, 299, 398; 20 blocks 406,
  // 405, 512; 2304 tokens back to 1536, 8 blocks, 8 heads of 64 (128 bytes): 26.1 whole, 24.0 in halves, 25.1 in quarters.
  int lpr = whole.D * esz / 16, parts = 1;
  const long long groups = 2ll * n_blocks * whole.kv_heads * a.n;
  while (lpr > 4 && groups * parts < (lpr > 8 ? 1024 : 192)) lpr /= 2, parts *= 2;
  const dim3 grid(2 * n_blocks, whole.kv_heads * parts, a.n);
#define XC_MOVE(L) \
  evict_move_kernel<L><<<grid, 512, 0, st>>>(a, (char*)whole.keys, (char*)whole.values, whole.shift, whole.kv_heads, parts, block_bytes)
  if (lpr == 32) XC_MOVE(32);
  else if (lpr == 16) XC_MOVE(16);
  else if (lpr == 8) XC_MOVE(8);
  else XC_MOVE(4);
#undef XC_MOVE
  return hipGetLastError();
}

}  // namespace xc
