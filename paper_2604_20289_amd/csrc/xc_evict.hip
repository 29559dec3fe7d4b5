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

// Which tokens a sequence keeps: the m-th largest weight of those that are
// neither among the first nor the last by a search over the digits of its
// order (11, 11, 10 bits, a histogram each), then one pass in order that ranks
// and lists the kept ones and moves their weights.  A workgroup a sequence.
constexpr int kSelThreads = 1024, kSelItems = 8, kSelWaves = kSelThreads / 64, kBins = 2048, kCopies = 8;
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(EvictArgs a, int shift) {
  const EvictSeq s = a.seqs[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int* kept = a.kept ? a.kept + s.number * a.kept_ld : nullptr;
  if (s.keep < 0) {
    for (int t = tid; t < s.tokens; t += kSelThreads) kept[t] = t;
    return;
  }
  __shared__ unsigned hist[kBins * kCopies];
  __shared__ int totals[2][kSelWaves];
  __shared__ int found[2];
  float* w = a.weights + s.number * a.ld;
  const int lo = a.sinks, hi = s.tokens - a.recent;
  int want = s.keep - a.sinks - a.recent;  // of them
  unsigned prefix = 0;                     // the digits found so far
  for (int pass = 0; pass < 3 && want > 0; ++pass) {
    const int bits = pass == 2 ? 10 : 11, low = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = 1 << bits;
    for (int i = tid; i < bins * kCopies; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int t0 = lo; t0 < hi; t0 += kSelThreads * kSelItems) {
      float x[kSelItems];
#pragma unroll
      for (int u = 0; u < kSelItems; ++u) {
        const int t = t0 + u * kSelThreads + tid;
        x[u] = t < hi ? w[t] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kSelItems; ++u) {
        const unsigned o = order_of(x[u]);
        if (t0 + u * kSelThreads + tid < hi && (pass == 0 || o >> (low + bits) == prefix))
          atomicAdd(&hist[(o >> low & (bins - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
      }
    }
    __syncthreads();
    // bins from the top: thread i has bins 2 i and 2 i + 1 counted from there
    int n[2] = {0, 0};
    for (int k = 0; k < 2; ++k) {
      const int bin = bins - 1 - (2 * tid + k);
      if (bin >= 0)
        for (int c = 0; c < kCopies; ++c) n[k] += (int)hist[bin * kCopies + c];
    }
    int sum = n[0] + n[1];
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o, 64);
      if (lane >= o) sum += v;
    }
    if (lane == 63) totals[0][wave] = sum;
    __syncthreads();
    int above = sum - n[0] - n[1];
    for (int i = 0; i < wave; ++i) above += totals[0][i];
    for (int k = 0; k < 2; ++k) {
      if (above < want && above + n[k] >= want) found[0] = bins - 1 - (2 * tid + k), found[1] = want - above;
      above += n[k];
    }
    __syncthreads();
    prefix = prefix << bits | (unsigned)found[0];
    want = found[1];
    __syncthreads();
  }
  const bool any = s.keep > a.sinks + a.recent;
  const int ties = want;  // of those as heavy as the lightest kept one, the first so many

  int tie0 = 0, kept0 = 0;  // before the tokens at hand
  for (int t0 = 0; t0 < s.tokens; t0 += kSelThreads * kSelItems) {
    float x[kSelItems];
    unsigned long long tie[kSelItems], sel[kSelItems];
    const int at = t0 + wave * 64 * kSelItems + lane;
#pragma unroll
    for (int u = 0; u < kSelItems; ++u) x[u] = at + u * 64 < s.tokens ? w[at + u * 64] : 0.f;
    int n = 0;
#pragma unroll
    for (int u = 0; u < kSelItems; ++u) {
      const int t = at + u * 64;
      tie[u] = __builtin_amdgcn_ballot_w64(any && t >= lo && t < hi && order_of(x[u]) == prefix);
      n += __popcll(tie[u]);
    }
    if (lane == 0) totals[0][wave] = n;
    __syncthreads();
    int rank = tie0;
    for (int i = 0; i < kSelWaves; ++i) {
      if (i < wave) rank += totals[0][i];
      tie0 += totals[0][i];
    }
    n = 0;
#pragma unroll
    for (int u = 0; u < kSelItems; ++u) {
      const int t = at + u * 64, mine = rank + __popcll(tie[u] & ((1ull << lane) - 1));
      const bool is_tie = tie[u] >> lane & 1, mid = t >= lo && t < hi;
      sel[u] = __builtin_amdgcn_ballot_w64(t < s.tokens &&
                                           (!mid || (any && (is_tie ? mine < ties : order_of(x[u]) > prefix))));
      rank += __popcll(tie[u]);
      n += __popcll(sel[u]);
    }
    if (lane == 0) totals[1][wave] = n;
    __syncthreads();
    int pos = kept0;
    for (int i = 0; i < kSelWaves; ++i) {
      if (i < wave) pos += totals[1][i];
      kept0 += totals[1][i];
    }
    // a kept token goes to its own place or a lower one, and all of this turn have been read
#pragma unroll
    for (int u = 0; u < kSelItems; ++u) {
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
  for (int t = s.keep + tid; t < s.tokens; t += kSelThreads) w[t] = 0.f;
}

// Kept tokens to their places, in keys or values of one head of one block: one
// workgroup in order, since places are filled that later tokens... lie behind:
// a token's new place is its old one or lower, so what is loaded ahead has not
// been written over, and what is written has been loaded by all.
template <int LPR>
__global__ __launch_bounds__(512) void evict_move_kernel(EvictArgs a, char* keys, char* values, int shift, long long block_bytes) {
  constexpr int ROWS = 512 / LPR, U = 4;
  const EvictSeq s = a.seqs[blockIdx.z];
  if (s.keep <= 0) return;
  const int h = blockIdx.y, kv = gridDim.y, c = threadIdx.x % LPR, in_page = (1 << shift) - 1;
  u32x4* base = reinterpret_cast<u32x4*>((blockIdx.x & 1 ? values : keys) + (blockIdx.x >> 1) * block_bytes);
  auto at_of = [&](int place) __attribute__((always_inline)) {
    return ((((long long)(place >> shift) * kv + h) << shift) + (place & in_page)) * LPR + c;
  };
  // tokens in pages before the last first one's stay
  const int sink_page = (s.first + min(a.sinks, s.keep)) >> shift << shift;
  for (int j0 = max(0, sink_page - s.first); j0 < s.keep; j0 += ROWS * U) {
    long long to[U];
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * ROWS + threadIdx.x / LPR;
      to[u] = -1;
      if (j < s.keep) {
        const int from = a.src[s.at + j], place = s.first + j;
        const int dst = (a.tables[s.to + (place >> shift)] << shift) + (place & in_page);
        if (from != dst) {
          to[u] = at_of(dst);
          x[u] = base[at_of(from)];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+v"(x[u]));
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u] >= 0) base[to[u]] = x[u];
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, const PageBuf& whole, int esz, int n_blocks, long long block_bytes, int most,
                        hipStream_t st) {
  evict_select_kernel<<<a.n, kSelThreads, 0, st>>>(a, whole.shift);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || most <= 0) return e;
  const dim3 grid(2 * n_blocks, whole.kv_heads, a.n);
#define XC_MOVE(L) evict_move_kernel<L><<<grid, 512, 0, st>>>(a, (char*)whole.keys, (char*)whole.values, whole.shift, block_bytes)
  const int lpr = whole.D * esz / 16;
  if (lpr == 32) XC_MOVE(32);
  else if (lpr == 16) XC_MOVE(16);
  else XC_MOVE(8);
#undef XC_MOVE
  return hipGetLastError();
}

}  // namespace xc
