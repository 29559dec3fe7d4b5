// Evictions: which tokens a sequence keeps, and their keys and values moved
// to its first places.
#include "xc_chunk.h"

#include "xc_internal.h"

#include <math.h>

#include <type_traits>

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

// Which tokens a sequence keeps: those of the m-th largest order and above,
// where the first and the last ones' is above all others.  A search over the
// order's digits (11, 11, 10 bits, a histogram each, until all of a digit's are
// wanted), then one pass that ranks and lists the kept ones and moves their
// weights.  A workgroup a sequence, each wave a run of its tokens: its time is
// latency, of LDS and of barriers, and one CU's instructions.  Up to 24 tokens a
// thread stay in registers, with their orders.  2304 tokens, 768 of them 0, take
// 6.8 us, 21060 with 7020 16.4; with a pass of two barriers for every 8 tokens a
// thread, and orders formed anew each time, 12 and 26.  256 threads are quicker
// than 1024 up to about 1000 tokens (a call for 2000 takes 21.3 and 19.3 us).
constexpr int kBins = 2048, kSelectFew = 1024;
struct Nothing {};
template <int THREADS, typename Sent>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a, int shift, Sent sent) {
  constexpr int WAVES = THREADS / 64, HELD = 24, ITEMS = 8, PER = kBins / THREADS;
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  // what came with the launch is passed on to the rows' kernel
  constexpr bool LITTLE = std::is_same<Sent, Little>::value;
  const char* words = LITTLE ? reinterpret_cast<const char*>(&sent) : reinterpret_cast<const char*>(a.seqs);
  const EvictSeq s = reinterpret_cast<const EvictSeq*>(words)[blockIdx.x];
  const int* tables = reinterpret_cast<const int*>(words + (reinterpret_cast<const char*>(a.tables) - reinterpret_cast<const char*>(a.seqs)));
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int* kept = a.kept ? a.kept + s.number * a.kept_ld : nullptr;
  if (LITTLE && tid == 0) a.seqs[blockIdx.x] = s;
  if (s.keep < 0) {
    for (int t = tid; t < s.tokens; t += THREADS) kept[t] = t;
    return;
  }
  if (LITTLE && s.keep > 0)
    for (int i = tid; i <= (s.first + s.keep - 1) >> shift; i += THREADS) a.tables[s.to + i] = tables[s.to + i];
  __shared__ __attribute__((aligned(16))) int hist[kBins][4];  // a copy for every fourth lane
  __shared__ int totals[2][WAVES];
  __shared__ int found[3], stays;
  __shared__ int pages[HELD * THREADS / 16 + 1];
  float* w = a.weights + s.number * a.ld;
  constexpr unsigned kAlways = ~0u;  // (of no weight)
  auto order_at = [&](float x, int t) __attribute__((always_inline)) {
    // behind the last token: 0, with the lightest, and behind all of them in every tie
    return t < s.tokens ? (t >= a.sinks && t < s.tokens - a.recent ? order_of(x) : kAlways) : 0u;
  };
  int want = s.keep - a.sinks - a.recent;  // of the others
  const bool held = s.tokens <= HELD * THREADS;
  const int span = (s.tokens + THREADS - 1) / THREADS * 64, mine = wave * span + lane;
  float own[HELD];
  unsigned order[HELD];
  if (held) {
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (u * 64 < span) own[u] = w[min(mine + u * 64, s.tokens - 1)];
    for (int i = tid; i <= (s.first + s.tokens - 1) >> shift; i += THREADS) pages[i] = tables[s.from + i];
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (u * 64 < span) order[u] = order_at(own[u], mine + u * 64);
  }
  unsigned prefix = 0;  // the digits found so far
  int below = 32;       // the bits behind them
  if (want == 0) prefix = kAlways - 1, below = 0;
  for (int pass = 0; pass < 3 && want > 0; ++pass) {
    const int bits = pass == 2 ? 10 : 11, low = below - bits;
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<i32x4*>(hist[i * THREADS + tid]) = i32x4{0, 0, 0, 0};
    __syncthreads();
    auto count = [&](unsigned o) __attribute__((always_inline)) {
      if (pass == 0 ? o != kAlways : o >> below == prefix) atomicAdd(&hist[o >> low & ((1 << bits) - 1)][lane & 3], 1);
    };
    if (held) {
#pragma unroll
      for (int u = 0; u < HELD; ++u)
        if (u * 64 < span) count(order[u]);
    } else {
      for (int t0 = 0; t0 < s.tokens; t0 += THREADS * ITEMS) {
        float x[ITEMS];
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) x[u] = w[min(t0 + u * THREADS + tid, s.tokens - 1)];
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) count(order_at(x[u], t0 + u * THREADS + tid));
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
  const unsigned long long lower = (1ull << lane) - 1;
  // lanes whose token is as heavy as the lightest kept one, and heavier
  struct Lanes {
    unsigned long long tie, more;
  };
  auto lanes_of = [&](unsigned o) __attribute__((always_inline)) {
    return Lanes{__builtin_amdgcn_ballot_w64(o >> below == prefix), __builtin_amdgcn_ballot_w64(o >> below > prefix)};
  };
  auto kept_of = [&](const Lanes& l, int rank) __attribute__((always_inline)) {
    const bool tie = l.tie >> lane & 1, more = l.more >> lane & 1;
    return __builtin_amdgcn_ballot_w64(more || (tie && rank + __popcll(l.tie & lower) < ties));
  };
  auto keep = [&](int t, int j, float x, int page) __attribute__((always_inline)) {
    const int place = s.first + t;
    a.src[s.at + j] = (page << shift) + (place & ((1 << shift) - 1));
    if (kept) kept[j] = t;
    w[j] = x;
  };
  // kept by the waves before this one, of ties (and all tokens) before the waves' at hand
  auto before = [&](int tie0, int& rank, int& pos, int& all_ties, int& all_kept) __attribute__((always_inline)) {
    const int tie = lane < WAVES ? totals[0][lane] : 0, tie_to = lanes_up_to(tie), tie_before = tie0 + tie_to - tie;
    const int n = (lane < WAVES ? totals[1][lane] : 0) + min(max(ties - tie_before, 0), tie), to = lanes_up_to(n);
    rank = __builtin_amdgcn_readlane(tie_before, wave);
    pos = __builtin_amdgcn_readlane(to - n, wave);
    all_ties = __builtin_amdgcn_readlane(tie_to, 63);
    all_kept = __builtin_amdgcn_readlane(to, 63);
  };
  int rank, pos, all_ties, all_kept, first = s.keep;  // first: of this wave's tokens, the first one not kept
  auto not_kept = [&](unsigned long long sel, int t0) __attribute__((always_inline)) {  // of the 64 from t0 on
    if (~sel) first = min(first, t0 + (int)__builtin_ctzll(~sel));
  };
  if (tid == 0) stays = s.keep;
  if (held) {
    int n_tie = 0, n_more = 0;
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (u * 64 < span) {
        const Lanes l = lanes_of(order[u]);
        n_tie += __popcll(l.tie), n_more += __popcll(l.more);
        asm volatile("" ::"v"(own[u]));  // (there before anything is written)
      }
    if (lane == 0) totals[0][wave] = n_tie, totals[1][wave] = n_more;
    __syncthreads();
    before(0, rank, pos, all_ties, all_kept);
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (u * 64 < span) {
        const Lanes l = lanes_of(order[u]);
        const unsigned long long sel = kept_of(l, rank);
        const int t = mine + u * 64;
        if (sel >> lane & 1) keep(t, pos + __popcll(sel & lower), own[u], pages[(s.first + t) >> shift]);
        not_kept(sel, wave * span + u * 64);
        rank += __popcll(l.tie);
        pos += __popcll(sel);
      }
  } else {
    int tie0 = 0, kept0 = 0;  // before the tokens at hand
    for (int t0 = 0; t0 < s.tokens; t0 += THREADS * ITEMS) {
      float x[ITEMS];
      Lanes l[ITEMS];
      const int at = t0 + wave * 64 * ITEMS + lane;
#pragma unroll
      for (int u = 0; u < ITEMS; ++u) x[u] = w[min(at + u * 64, s.tokens - 1)];
      int n_tie = 0, n_more = 0;
#pragma unroll
      for (int u = 0; u < ITEMS; ++u) {
        l[u] = lanes_of(order_at(x[u], at + u * 64));
        n_tie += __popcll(l[u].tie), n_more += __popcll(l[u].more);
        asm volatile("" ::"v"(x[u]));
      }
      if (lane == 0) totals[0][wave] = n_tie, totals[1][wave] = n_more;
      __syncthreads();
      before(tie0, rank, pos, all_ties, all_kept);
      pos += kept0;
      tie0 += all_ties, kept0 += all_kept;
      // a kept token goes to its own place or a lower one, and all of this turn have been read
#pragma unroll
      for (int u = 0; u < ITEMS; ++u) {
        const unsigned long long sel = kept_of(l[u], rank);
        const int t = at + u * 64;
        if (sel >> lane & 1) keep(t, pos + __popcll(sel & lower), x[u], tables[s.from + ((s.first + t) >> shift)]);
        not_kept(sel, t0 + wave * 64 * ITEMS + u * 64);
        rank += __popcll(l[u].tie);
        pos += __popcll(sel);
      }
      __syncthreads();  // (totals have been read)
    }
  }
  if (lane == 0 && first < s.keep) atomicMin(&stays, first);
  for (int t = s.keep + tid; t < s.tokens; t += THREADS) w[t] = 0.f;
  __syncthreads();
  if (tid == 0) a.stays[blockIdx.x] = stays;
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
  // tokens before the first one given up stay, but for replaced pages: there those of pages of nothing but first tokens
  const int sink_page = (s.first + min(a.sinks, s.keep)) >> shift << shift;
  const int j0 = s.replaced ? max(0, sink_page - s.first) : a.stays[blockIdx.z];
  if (j0 >= s.keep) return;
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

hipError_t launch_evict(const EvictArgs& a, const Little* little, const PageBuf& whole, int esz, int n_blocks,
                        long long block_bytes, int most_tokens, int most, hipStream_t st) {
  if (most_tokens <= kSelectFew) {
    if (little) evict_select_kernel<256><<<a.n, 256, 0, st>>>(a, whole.shift, *little);
    else evict_select_kernel<256><<<a.n, 256, 0, st>>>(a, whole.shift, Nothing{});
  } else {
    if (little) evict_select_kernel<1024><<<a.n, 1024, 0, st>>>(a, whole.shift, *little);
    else evict_select_kernel<1024><<<a.n, 1024, 0, st>>>(a, whole.shift, Nothing{});
  }
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
