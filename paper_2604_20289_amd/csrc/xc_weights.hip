// The weight that the rows of a batch give to each token of their sequences:
// w_j = decay w_j + sum over rows and heads of exp(scale q k_j - lse).
//
// S^T = K Q^T on the matrix cores, as in the attention, but a wave keeps its
// keys' operand in registers and the queries go by: every sum over rows is a
// lane's own until the end.  Nothing is added by atomics, and every sum has a
// fixed order.  exp2(x - hi) f, with lse log2(e) = hi + lo rounded apart and f =
// 2^-lo, keeps what the product with log2(e) would lose of a large lse.
//
// Two kinds of workgroup.  Many rows: weights_kernel (float32, of few rows too:
// weights_f32_kernel), 256 (128) keys of one head against a run of rows, whose
// partial sums weights_join_kernel adds up.  bf16 batches of sequences that all
// have few rows: weights_few_kernel, all heads of a few keys, read once for all
// sequences that have them.
#include "xc_chunk.h"

#include "xc_internal.h"
#include "xc_tiles.h"

#include <math.h>

#include <type_traits>

namespace xc {

namespace {

// exp(x ln 2 - lse) = exp2(x - hi) * f
struct Term {
  float hi, f;
};
__device__ __forceinline__ Term term_of(float lse) {
  constexpr float kLog2e = 1.44269502162933349609375f, kRest = 1.925963033500e-8f;
  const float hi = lse * kLog2e, lo = __builtin_fmaf(lse, kLog2e, -hi) + lse * kRest;
  // Infinite or NaN: hi says it.  From some 10^9 on lo itself is past 128: bounded, so that f is a number and nothing times f
  // nothing.
  return {hi, lo == lo ? __builtin_amdgcn_exp2f(__builtin_amdgcn_fmed3f(-lo, -126.f, 126.f)) : 1.f};
}

// (nothing, where it is no row)
__device__ __forceinline__ Limits limits_of(const ChunkSeq& q, const ChunkMask& m, int r, bool row) {
  const Seen w = seen(q, m, r);
  return {w.begin, row ? w.end : w.begin, q.first, row ? w.sink_end : q.first};
}

// Element i of a lane's 16 scores: the key's place among the 32 of its half
// tile, less 4 in the upper half wave.
__device__ __forceinline__ int key_of(int i) { return (i >> 2) * 8 + (i & 3); }

__device__ __forceinline__ unsigned keep_bit(unsigned bits, int at) { return (unsigned)((int)(bits << (31 - at)) >> 31); }

// 4 bytes per lane, global -> LDS
__device__ __forceinline__ void dma4(const char* base, unsigned off, char* lds) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), (short)0, -1, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds, 4, (int)off, 0, 0, 0);
}

// A unit's query rows: query row i is query head i % group of the unit's token i / group.
struct QueryRows {
  int n, group;
  unsigned by_group;
  __device__ __forceinline__ int token(int i) const { return (int)__umulhi((unsigned)i, by_group) + (group == 1 ? i : 0); }
  __device__ __forceinline__ int clamped(int i) const { return min(i, n - 1); }
};

// Sum over the 32 lanes of a half wave of 16 numbers each: lane l (of 16) of the
// lower (upper) row of 16 lanes gets number l (8 + l), l < 8.
__device__ __forceinline__ float fold(const f32x16& v, int lane) {
  float x[8], out = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 8]), false, false);
    x[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    auto add = [&](auto ctrl) __attribute__((always_inline)) {
      x[i] += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x[i]), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    add(std::integral_constant<int, 0xB1>{});   // lane ^ 1
    add(std::integral_constant<int, 0x4E>{});   // lane ^ 2
    add(std::integral_constant<int, 0x141>{});  // the two quads of 8 lanes
    add(std::integral_constant<int, 0x140>{});  // the two halves of a row of 16
    if ((lane & 15) == i) out = x[i];
  }
  return out;
}

// 4 waves of 64 keys.  The queries come by in stages of 64 rows through a ring
// of four.  Products of a tile of 32 rows and exponentials of the one before
// alternate, two (d = 64: four) to a product, so that the matrix units and the
// others work at once (a step of one product, two exponentials and four
// multiply-adds takes 41 cycles of a SIMD with two such waves, where the product
// alone takes 32 and the others 30).  Two workgroups per CU, three at d = 64.
//
// Bound by both: 7020 rows, 21060 keys, 12 heads of 128 take 450 us, 1010
// TFLOP/s, with the products alone 341 and without them 333, at 2.0 GHz and
// 87% of the wave slots; at d = 64 the exponentials: 16384 rows of 8
// sequences, 6144 keys, 8 heads 140 us.  Tried: a tile's products, then its
// exponentials, with the other wave of the SIMD in the other phase by chance,
// 482 us; 32 keys a wave and four waves per SIMD 478; workgroups of 512 keys 463;
// two stages instead of four 470.  An unrolled ring with an array per slot spills.
template <int D>
__global__ __launch_bounds__(256, 2) void weights_kernel(WeightArgs a) {
  using F = Frags<D>;
  constexpr int KCG = F::KCG, KS = F::KS, SLOT = 64 * D * 2, NB = 2 * KCG;  // blocks of a stage per wave
  constexpr int TERMS = 4 * 64 * 4;  // each wave's copy of a stage's log-sum-exps
  // queries, then log-sum-exps; one array and no other, in which the compiler leaves it to the waits here what has landed
  __shared__ __attribute__((aligned(1024))) char ring[4 * (SLOT + TERMS)];
  int u, h;
  if (!xcd_pair(blockIdx.x, a.n_units, a.n_long, a.buf.kv_heads, u, h)) return;
  const WeightUnit un = a.units[u];
  const ChunkSeq sq = a.seqs[un.seq];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const QueryRows rows{(un.r1 - un.r0) * a.group, a.group, a.by_group};
  const int n = (rows.n + 63) >> 6;
  const long long ld = a.q_ld * 2;
  const char* q = reinterpret_cast<const char*>(a.q) + (long long)(sq.row0 + un.r0) * ld + (long long)h * a.group * D * 2;
  const char* lse = reinterpret_cast<const char*>(a.lse + (long long)(sq.row0 + un.r0) * a.q_heads + h * a.group);

  // What a lane fetches of a stage lies as far from the stage's first token in every whole one, where 64 rows are whole
  // tokens (group divides 64).
  unsigned q_off[NB], l_off;
  auto offsets = [&](int at) __attribute__((always_inline)) {
    const int first = rows.token(rows.clamped(at));
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int B = wave + 4 * i, rg = B / KCG, cg = B % KCG;
      const int t0 = rows.token(rows.clamped(at + rg * 8));
      const int r = rows.clamped(at + rg * 8 + ((lane >> 3) ^ (rg & 1))), t = rows.token(r);
      q_off[i] = (unsigned)(t - t0) * (unsigned)ld + (r - t * a.group) * (D * 2) + k_block_col(rg, cg, lane);
    }
    const int r = rows.clamped(at + lane), t = rows.token(r);
    l_off = ((t - first) * a.q_heads + r - t * a.group) * 4;
  };
  const bool whole = (a.group & (a.group - 1)) == 0 && a.group <= 64;
  offsets(0);
  auto request = [&](int s) __attribute__((always_inline)) {
    const int at = min(s, n - 1) * 64;  // past the last stage that one again: as many in flight as ever
    if (!whole || at + 64 > rows.n) offsets(at);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int B = wave + 4 * i;
      dma16(q + rows.token(rows.clamped(at + B / KCG * 8)) * ld, q_off[i], ring + (s & 3) * SLOT + B * 1024);
    }
    dma4(lse + (long long)rows.token(at) * a.q_heads * 4, l_off, ring + 4 * SLOT + (s & 3) * TERMS + wave * 256);
  };
  request(0);
  request(1);
  request(2);

  const int k0 = un.lo + wave * 64;
  bf16x8 kf[2][KS];
#pragma unroll
  for (int mt = 0; mt < 2; ++mt) {
    const int at = min(k0 + mt * 32 + lo, un.hi - 1);
    const long long page = a.tables[sq.table + (at >> a.buf.shift)];
    const bf16* k = reinterpret_cast<const bf16*>(a.buf.keys) +
                    (((page * a.buf.kv_heads + h) << a.buf.shift) + (at & ((1 << a.buf.shift) - 1))) * D + hi * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[mt][ks] = *reinterpret_cast<const bf16x8*>(k + ks * 16);
  }
  // tiles [free0, free1) of 32 query rows see all of this wave's keys
  const RowRange all = rows_seeing_all(sq, a.mask, min(k0, un.hi - 1), min(k0 + 64, un.hi));
  const RowRange free = tiles_within(all, un.r0, un.r1, a.group);
  const int free0 = __builtin_amdgcn_readfirstlane(free.begin), free1 = __builtin_amdgcn_readfirstlane(free.end);
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(kf[mt][ks]));

  f32x16 sa[2], sb[2], acc[2];
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) sb[mt][i] = -INFINITY, acc[mt][i] = 0.f;
  Term ta, tb{0.f, 0.f};
  const F f(lane);
  // a tile that hides something: what is hidden weighs nothing, whatever the row's sum is; one that is no finite number
  // goes where the row sees
  auto masked = [&](int number, f32x16 (&s)[2], Term& t) __attribute__((always_inline)) {
    if (number < 0 || (number >= free0 && number < free1)) return;
    const int r = number * 32 + lo;
    const Limits lim = limits_of(sq, a.mask, un.r0 + rows.token(rows.clamped(r)), r < rows.n);
    const bool finite = fabsf(t.hi) < INFINITY;
    const float other = -t.hi;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const unsigned bits = lim.bits(k0 + mt * 32) >> (hi * 4);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[mt][i] = finite ? s[mt][i] : other;
      mask_row(s[mt], bits, key_of);
    }
    if (!finite) t = {0.f, 1.f};
  };
  // products of a tile (its half of the stage in slot) with the exponentials of the one before
  auto tile = [&](const char* slot, int half, f32x16 (&s)[2], const f32x16 (&before)[2], const Term& t) __attribute__((always_inline)) {
    constexpr int PF = 4, STEPS = 2 * KS, EACH = 32 / STEPS;
    bf16x8 fr[PF];
#pragma unroll
    for (int i = 0; i < PF; ++i) fr[i] = f.k(slot, half, i);
    float arg[EACH], e[EACH];
    auto score = [&](int x) __attribute__((always_inline)) { return before[x >> 4][x & 15]; };
#pragma unroll
    for (int k = 0; k < EACH; ++k) arg[k] = __builtin_fmaf(score(k), a.scale, -t.hi);
    // a step: a product, the exponentials of one group of scores, the next one's arguments, the sums of the last one
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int mt = i & 1, ks = i >> 1;
      if (ks == 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[mt][r] = 0.f;
      }
      s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[mt][ks], fr[ks % PF], s[mt], 0, 0, 0);
      if (mt == 1 && ks + PF < KS) fr[ks % PF] = f.k(slot, half, ks + PF);
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        const int x = i * EACH + k;
        if (i > 0) acc[(x - EACH) >> 4][(x - EACH) & 15] = __builtin_fmaf(e[k], t.f, acc[(x - EACH) >> 4][(x - EACH) & 15]);
        e[k] = __builtin_amdgcn_exp2f(arg[k]);
        if (i + 1 < STEPS) arg[k] = __builtin_fmaf(score(x + EACH), a.scale, -t.hi);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int x = (STEPS - 1) * EACH + k;
      acc[x >> 4][x & 15] = __builtin_fmaf(e[k], t.f, acc[x >> 4][x & 15]);
    }
    // ... all of it here: without this the compiler moves the exponentials behind the next tile's products
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) asm volatile("" : "+v"(acc[mt]));
  };
  for (int s = 0; s < n; ++s) {
    const char* slot = ring + (s & 3) * SLOT;
    XC_WAIT_VM(2 * (NB + 1));  // all but stages s + 1 and s + 2
    tile_barrier();  // this stage is there, and the one before has been read
    request(s + 3);
    const float* l = reinterpret_cast<const float*>(ring + 4 * SLOT + (s & 3) * TERMS + wave * 256);
    const float la = l[lo], lb = l[32 + lo];
    masked(2 * s - 1, sb, tb);
    tile(slot, 0, sa, sb, tb);
    ta = term_of(la);
    masked(2 * s, sa, ta);
    tile(slot, 1, sb, sa, ta);
    tb = term_of(lb);
  }
  XC_WAIT_VM(0);
  masked(2 * n - 1, sb, tb);
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      acc[mt][i] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(sb[mt][i], a.scale, -tb.hi)), tb.f, acc[mt][i]);
  float* to = a.parts + ((long long)un.part * a.buf.kv_heads + h) * kWeightKeys + wave * 64;
#pragma unroll
  for (int mt = 0; mt < 2; ++mt) {
    const float x = fold(acc[mt], lane);
    const int i = (lane & 7) + ((lane >> 4) & 1) * 8;
    if ((lane & 15) < 8) to[mt * 32 + key_of(i) + hi * 4] = x;
  }
}

// float32: 4 waves of 32 keys, stages of 32 rows, v_mfma_f32_32x32x2_f32 (both k
// indices of a product are head dims 8 t + e and 8 t + 4 + e, as in the
// attention).  Bound by these products.
template <int D>
__global__ __launch_bounds__(256) void weights_f32_kernel(WeightArgs a) {
  constexpr int CH = D / 4, SLOT = 32 * D * 4, NB = SLOT / 4096, RPB = 64 / CH;  // 16-byte chunks of a row, rows of a 1 KB block
  constexpr int TERMS = 4 * 64 * 4;
  __shared__ __attribute__((aligned(1024))) char ring[4 * (SLOT + TERMS)];  // as above
  int u, h;
  if (!xcd_pair(blockIdx.x, a.n_units, a.n_long, a.buf.kv_heads, u, h)) return;
  const WeightUnit un = a.units[u];
  const ChunkSeq sq = a.seqs[un.seq];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const QueryRows rows{(un.r1 - un.r0) * a.group, a.group, a.by_group};
  const int n = (rows.n + 31) >> 5;
  const long long ld = a.q_ld * 4;
  const char* q = reinterpret_cast<const char*>(a.q) + (long long)(sq.row0 + un.r0) * ld + (long long)h * a.group * D * 4;
  const char* lse = reinterpret_cast<const char*>(a.lse + (long long)(sq.row0 + un.r0) * a.q_heads + h * a.group);
  auto swz = [](int r, int c) __attribute__((always_inline)) {
    return c ^ (CH >= 16 ? (r & 7) ^ ((r & 4) << 1) : r & 7);
  };
  auto request = [&](int s) __attribute__((always_inline)) {
    const int at = min(s, n - 1) * 32;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int B = wave + 4 * i, row = B * RPB + lane / CH;
      const int t0 = rows.token(rows.clamped(at + B * RPB)), r = rows.clamped(at + row), t = rows.token(r);
      dma16(q + t0 * ld, (unsigned)(t - t0) * (unsigned)ld + (r - t * a.group) * (D * 4) + swz(row, lane % CH) * 16,
            ring + (s & 3) * SLOT + B * 1024);
    }
    const int t0 = rows.token(rows.clamped(at)), r = rows.clamped(at + lo), t = rows.token(r);
    dma4(lse + (long long)t0 * a.q_heads * 4, ((t - t0) * a.q_heads + r - t * a.group) * 4,
         ring + 4 * SLOT + (s & 3) * TERMS + wave * 256);
  };
  request(0);
  request(1);
  request(2);
  const int k0 = un.lo + wave * 32;
  f32x4 kf[D / 8];
  {
    const int at = min(k0 + lo, un.hi - 1);
    const long long page = a.tables[sq.table + (at >> a.buf.shift)];
    const float* k = reinterpret_cast<const float*>(a.buf.keys) +
                     (((page * a.buf.kv_heads + h) << a.buf.shift) + (at & ((1 << a.buf.shift) - 1))) * D + hi * 4;
#pragma unroll
    for (int t = 0; t < D / 8; ++t) kf[t] = *reinterpret_cast<const f32x4*>(k + t * 8);
  }
  const RowRange all = rows_seeing_all(sq, a.mask, min(k0, un.hi - 1), min(k0 + 32, un.hi));
  const RowRange free = tiles_within(all, un.r0, un.r1, a.group);
  const int free0 = __builtin_amdgcn_readfirstlane(free.begin), free1 = __builtin_amdgcn_readfirstlane(free.end);
#pragma unroll
  for (int t = 0; t < D / 8; ++t) asm volatile("" : "+v"(kf[t]));
  f32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  for (int st = 0; st < n; ++st) {
    const char* slot = ring + (st & 3) * SLOT;
    XC_WAIT_VM(2 * (NB + 1));
    tile_barrier();
    request(st + 3);
    const Term t = term_of(reinterpret_cast<const float*>(ring + 4 * SLOT + (st & 3) * TERMS + wave * 256)[lo]);
    f32x16 s, o;  // two sums: no product waits for the one before it
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = o[i] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(slot + lo * (D * 4) + swz(lo, j * 2 + hi) * 16);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j][e], x[e], s, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j][e + 1], x[e + 1], o, 0, 0, 0);
      }
    }
    unsigned bits = ~0u;
    if (st < free0 || st >= free1) {
      const int r = st * 32 + lo;
      const Limits lim = limits_of(sq, a.mask, un.r0 + rows.token(rows.clamped(r)), r < rows.n);
      bits = lim.bits(k0) >> (hi * 4);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i] + o[i], a.scale, -t.hi));
      acc[i] = __builtin_fmaf(__uint_as_float(__float_as_uint(e) & keep_bit(bits, key_of(i))), t.f, acc[i]);
    }
  }
  XC_WAIT_VM(0);
  const float x = fold(acc, lane);
  const int i = (lane & 7) + ((lane >> 4) & 1) * 8;
  if ((lane & 15) < 8)
    a.parts[((long long)un.part * a.buf.kv_heads + h) * kWeightKeysF32 + wave * 32 + key_of(i) + hi * 4] = x;
}

// Partial sums of a tile of keys, in a fixed order: 1024 threads, as many to a
// key as there are, each every so many of its sums.
template <int KEYS>
__global__ __launch_bounds__(1024) void weights_join_kernel(WeightArgs a) {
  constexpr int N = 1024 / KEYS;
  __shared__ float sums[N][KEYS];
  const WeightTile t = a.tiles[blockIdx.x];
  const ChunkSeq q = a.seqs[t.seq];
  const int k = threadIdx.x % KEYS, g = threadIdx.x / KEYS, parts = t.parts * a.buf.kv_heads;
  const float* from = a.parts + (long long)t.part * a.buf.kv_heads * KEYS + k;
  float* to = a.weights + q.number * a.ld + (t.lo - q.first + k);
  const bool mine = g == 0 && t.lo + k < t.hi;
  const float old = mine && a.decay != 0.f ? *to * a.decay : 0.f;
  float sum = 0.f;
  int i = g;
  for (; i + 3 * N < parts; i += 4 * N) {
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = from[(long long)(i + j * N) * KEYS];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += x[j];
  }
  for (; i < parts; i += N) sum += from[(long long)i * KEYS];
  sums[g][k] = sum;
  __syncthreads();
  if (!mine) return;
  sum = sums[0][k];
#pragma unroll
  for (int j = 1; j < N; ++j) sum += sums[j][k];
  *to = old + sum;
}

// Few rows: a workgroup has a tile of keys (or 2 or 4 of them, with 2 or 3 key
// heads or one) and its waves share the heads; each has two K tiles in LDS, one
// on its way.  A lane has a query row of every head, so its sums of 16 keys go on
// over all heads; then they meet in LDS, the rows of each sequence and the
// waves' shares.  What a row does not see is left out there, once for all heads.
//
// All that a workgroup has to know comes in two steps (its run, then rows,
// pages and where its sums go), so that keys, queries and the old sums are asked
// for together: 12.6 us for 16 rows over 14040 shared keys and 100 of their own,
// 12 heads of 128 (48 MB), where a search for the run and each row's sequence one
// after the other take 14.4; 6.8 instead of 7.9 over 200 keys.
// The rows of a sequence are summed by one lane of each key, by 2 to 8 where there
// are few outputs of many rows (64 rows of one sequence over 4000 keys: 21.8 us
// with one, 11.7), and the old sums of further outputs are asked for four at a
// time (64 sequences over 20000 keys, 8 heads of 64: 29.1 us one by one, 27.0).
// Bound by latency and by reading keys: one row over 48448 keys, 16 heads of 128
// (198 MB) 31 us; 64 rows over 36288 and 100, 16 heads, 71, of which the queries
// are much: a row per lane, 64 lines a load.  (By DMA into LDS, as the keys, they
// gain nothing for 16 rows and lose a third for 64, whose LDS then leaves room for
// one workgroup.)
template <int D, int G>
__device__ __forceinline__ void few_weights(const WeightArgs& a, const WeightFew& run, char* ring) {
  using F = Frags<D>;
  constexpr int KCG = F::KCG, KS = F::KS, KEYS = few_keys(D), HT = KEYS / 32, TILE = KEYS * D * 2, LOADS = TILE / 1024, R = 32 * G;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const int kv = a.buf.kv_heads, hw = few_head_waves(kv), h0 = wave % hw;
  const int in_page = (1 << a.buf.shift) - 1, last = run.hi - 1, group_keys = KEYS * 4 / hw;
  const int group0 = (run.lo & ~15) + (blockIdx.x - run.group0) * group_keys, at0 = group0 + wave / hw * KEYS;
  const QueryRows rows{run.rows * a.group, a.group, a.by_group};

  // what this lane's rows see
  int token[G];
  WeightInfo row[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    token[g] = rows.token(rows.clamped(g * 32 + lo));
    row[g] = a.infos[run.info + token[g]];
  }
  // The first sums that this thread is to write: where, and what is there (asked for with the first keys).
  struct Out {
    float* to;
    float old;
    int rows;  // of the first row and past the last, 8 bits each
  };
  // Where they are few and of many rows, 2, 4 or 8 neighbouring lanes have one, each every so many of its rows.
  const int n_out = run.seqs * group_keys;
  const int lanes_log2 = rows.n < 8 * run.seqs ? 0 : n_out <= 32 ? 3 : n_out <= 64 ? 2 : n_out <= 128 ? 1 : 0;
  auto out_of = [&](int x) __attribute__((always_inline)) {
    const int o = x >> lanes_log2, si = min(o, n_out - 1) >> __builtin_ctz(group_keys), at = group0 + o - si * group_keys;
    const WeightInfo s = a.infos[run.info + run.rows + si];
    const bool is = o < n_out && at >= run.lo && at <= last;
    return Out{is ? a.weights + s.a * a.ld + (at - run.first) : nullptr, 0.f, s.b | s.c << 8};
  };
  auto old_of = [&](Out& o) __attribute__((always_inline)) {
    if (a.decay != 0.f && o.to) o.old = *o.to * a.decay;
  };
  constexpr int AHEAD = 3 - G;
  constexpr bool LATE = G * HT > 2;  // (no registers for them)
  Out out[AHEAD];
  if (!LATE) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) out[i] = out_of(threadIdx.x + i * 256);
  }

  // the groups of 16 places, each in one page; places outside the run read the nearest of it
  long long page_at[KEYS / 16];
  unsigned row_at[KEYS / 8];
  const long long head_bytes = (long long)D * 2 << a.buf.shift;
#pragma unroll
  for (int j = 0; j < KEYS / 16; ++j) {
    const int g0 = min(max(at0 + j * 16, run.lo), last);
    const long long page = a.tables[run.table + (g0 >> a.buf.shift)];
    page_at[j] = page * kv * head_bytes;
  }
#pragma unroll
  for (int rg = 0; rg < KEYS / 8; ++rg) {
    const int at = min(max(at0 + rg * 8 + ((lane >> 3) ^ (rg & 1)), run.lo), last);
    row_at[rg] = (unsigned)(at & in_page) * (D * 2) + k_block_col(rg, 0, lane);
  }
  char* kt = ring + wave * (2 * TILE);
  auto request = [&](int i) __attribute__((always_inline)) {
    const char* keys = reinterpret_cast<const char*>(a.buf.keys) + (h0 + i * hw) * head_bytes;
#pragma unroll
    for (int rg = 0; rg < KEYS / 8; ++rg)
#pragma unroll
      for (int cg = 0; cg < KCG; ++cg)
        dma16(keys + page_at[rg >> 1], row_at[rg] + cg * 128, kt + (i & 1) * TILE + (rg * KCG + cg) * 1024);
  };
  auto bits_of = [&](int g, int at) __attribute__((always_inline)) {
    const unsigned b = Limits{row[g].a, row[g].b, run.first, row[g].c}.bits(at);
    return g * 32 + lo < rows.n ? b : 0u;
  };
  // without a window every tile is seen
  bool any = false;
  if (a.mask.window != ChunkMask::kNone) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int mt = 0; mt < HT; ++mt) any |= bits_of(g, at0 + mt * 32) != 0;
  } else {
    any = true;
  }
  const int n = at0 <= last && __builtin_amdgcn_ballot_w64(any) != 0 ? (kv - h0 + hw - 1) / hw : 0;  // heads h0, h0 + hw, ..

  bf16x8 q[2][G][KS];
  float l[2][G];
  auto queries = [&](int i, bf16x8 (&x)[G][KS], float (&y)[G]) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int r = rows.clamped(g * 32 + lo), head = (h0 + i * hw) * a.group + r - rows.token(r) * a.group;
      const bf16* p = reinterpret_cast<const bf16*>(a.q) + (run.row0 + token[g]) * a.q_ld + (long long)head * D + hi * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x[g][ks] = *reinterpret_cast<const bf16x8*>(p + ks * 16);
      y[g] = a.lse[(long long)(run.row0 + token[g]) * a.q_heads + head];
    }
  };
  f32x16 acc[G][HT];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int mt = 0; mt < HT; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[g][mt][i] = 0.f;
  const F f(lane);
  // head i, while the next one's (unless it is the last) keys and queries come
  auto head = [&](int i, auto last, bf16x8 (&x)[G][KS], float (&y)[G], bf16x8 (&nx)[G][KS], float (&ny)[G]) __attribute__((always_inline)) {
    if constexpr (!last) {
      request(i + 1);
      queries(i + 1, nx, ny);
      asm volatile("" ::: "memory");  // (all of them before the wait that counts them)
      XC_WAIT_VM(LOADS + G * (KS + 1));
    } else {
      XC_WAIT_VM(0);
    }
    asm volatile("" ::: "memory");
    const char* tile = kt + (i & 1) * TILE;
    f32x16 s[G][HT];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int mt = 0; mt < HT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[g][mt][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int mt = 0; mt < HT; ++mt) {
        const bf16x8 k = f.k(tile, mt, ks);
#pragma unroll
        for (int g = 0; g < G; ++g) s[g][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, x[g][ks], s[g][mt], 0, 0, 0);
      }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const Term t = term_of(y[g]);
#pragma unroll
      for (int mt = 0; mt < HT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          acc[g][mt][r] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[g][mt][r], a.scale, -t.hi)), t.f, acc[g][mt][r]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this tile has been read
  };
  if (n > 0) {
    request(0);
    queries(0, q[0], l[0]);
  }
  if (!LATE) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) old_of(out[i]);
  }
  constexpr std::false_type more{};
  constexpr std::true_type last_one{};
  int i = 0;
  for (; i + 2 < n; i += 2) {
    head(i, more, q[0], l[0], q[1], l[1]);
    head(i + 1, more, q[1], l[1], q[0], l[0]);
  }
  if (i + 2 == n) {
    head(i, more, q[0], l[0], q[1], l[1]);
    head(i + 1, last_one, q[1], l[1], q[0], l[0]);
  } else if (i + 1 == n) {
    head(i, last_one, q[0], l[0], q[1], l[1]);
  }
  // key k, row r at k * R + (r + k) % R: lanes of different rows (written) or keys (read) meet different banks
  XC_WAIT_VM(0);
  float* mine = reinterpret_cast<float*>(kt);
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int mt = 0; mt < HT; ++mt) {
      const unsigned bits = bits_of(g, at0 + mt * 32) >> (hi * 4);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k = mt * 32 + key_of(i) + hi * 4;
        mine[k * R + ((g * 32 + lo + k) & (R - 1))] = __uint_as_float(__float_as_uint(acc[g][mt][i]) & keep_bit(bits, key_of(i)));
      }
    }
  __syncthreads();
  if (LATE) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) out[i] = out_of(threadIdx.x + i * 256), old_of(out[i]);
  }
  // rows from, from + step, .. of an output's, all waves' shares
  auto sum_of = [&](const Out& o, int gk, int from, int step) __attribute__((always_inline)) {
    const int k = gk % KEYS;
    float sum = 0.f;
    for (int w = 0; w < hw; ++w) {
      const float* part = reinterpret_cast<const float*>(ring + (gk / KEYS * hw + w) * (2 * TILE)) + k * R;
      for (int r = (o.rows & 255) + from; r < o.rows >> 8; r += step) sum += part[(r + k) & (R - 1)];
    }
    return sum;
  };
  if (lanes_log2 > 0) {
    const int lanes = 1 << lanes_log2, from = threadIdx.x & (lanes - 1);
    float sum = sum_of(out[0], threadIdx.x >> lanes_log2 & (group_keys - 1), from, lanes);
    auto add = [&](auto ctrl) __attribute__((always_inline)) {
      sum += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, sum), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    add(std::integral_constant<int, 0xB1>{});                  // lane ^ 1
    if (lanes > 2) add(std::integral_constant<int, 0x4E>{});   // lane ^ 2
    if (lanes > 4) add(std::integral_constant<int, 0x141>{});  // the two quads of 8 lanes
    if (out[0].to && from == 0) *out[0].to = out[0].old + sum;
    return;
  }
  auto write = [&](const Out& o, int x) __attribute__((always_inline)) {
    if (o.to) *o.to = o.old + sum_of(o, x & (group_keys - 1), 0, 1);
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) write(out[i], threadIdx.x + i * 256);
  // the others, so many at a time that their loads go together
  constexpr int BATCH = 4;
  for (int x = threadIdx.x + AHEAD * 256; x < n_out; x += BATCH * 256) {
    Out o[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) o[i] = out_of(x + i * 256);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) old_of(o[i]);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) write(o[i], x + i * 256);
  }
}
template <int D>
__global__ __launch_bounds__(256, 2) void weights_few_kernel(WeightArgs a) {
  __shared__ __attribute__((aligned(1024))) char ring[4 * 2 * few_keys(D) * D * 2];  // (one array and no other, as above)
  // its run is the last that begins at this workgroup or before: a lane each, 64 of them at a time
  int i = 0;
  for (int n = (a.n_runs + 63) / 64; n > 1;) {
    const int half = n / 2;
    if (a.runs[i + half * 64].group0 <= (int)blockIdx.x) i += half * 64, n -= half;
    else n = half;
  }
  const WeightFew mine = a.runs[min(i + (int)(threadIdx.x & 63), a.n_runs - 1)];
  const bool before = i + (int)(threadIdx.x & 63) < a.n_runs && mine.group0 <= (int)blockIdx.x;
  const int at = __popcll(__builtin_amdgcn_ballot_w64(before)) - 1;
  auto of = [&](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(x, at); };
  const WeightFew run{of(mine.group0), of(mine.lo),   of(mine.hi),   of(mine.table), of(mine.first),
                      of(mine.row0),   of(mine.rows), of(mine.seqs), of(mine.info)};
  if (run.rows * a.group > 32) few_weights<D, 2>(a, run, ring);
  else few_weights<D, 1>(a, run, ring);
}

}  // namespace

// Requirements (the caller's): D in {64, 128} (float32: 32 too); a row of q is shorter than 2^28 bytes; units and runs
// name rows, places and partial sums that there are.
hipError_t launch_weights(int dtype, const WeightArgs& a, hipStream_t st) {
  const int D = a.buf.D;
  if (a.n_runs > 0) {
    if (D == 128) weights_few_kernel<128><<<a.n_groups, 256, 0, st>>>(a);
    else weights_few_kernel<64><<<a.n_groups, 256, 0, st>>>(a);
    return hipGetLastError();
  }
  const unsigned grid = (unsigned)xcd_grid(a.n_units, a.buf.kv_heads);
  if (a.n_units > 0) {
    if (dtype == 1) {
      if (D == 128) weights_kernel<128><<<grid, 256, 0, st>>>(a);
      else weights_kernel<64><<<grid, 256, 0, st>>>(a);
    } else {
      if (D == 128) weights_f32_kernel<128><<<grid, 256, 0, st>>>(a);
      else if (D == 64) weights_f32_kernel<64><<<grid, 256, 0, st>>>(a);
      else weights_f32_kernel<32><<<grid, 256, 0, st>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (dtype == 1) weights_join_kernel<kWeightKeys><<<a.n_tiles, 1024, 0, st>>>(a);
  else weights_join_kernel<kWeightKeysF32><<<a.n_tiles, 1024, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace xc
