// Attention of branching sequences over paged keys and values:
// o = softmax(scale q k^T) v over all keys of the row's sequence.
//
// The work is cut on the host (plan_attention): a unit is up to tile_rows query
// rows over a run of keys of one page table.  The rows of a unit are (batch
// row, query head of one key head); for a shared history they come from many
// sequences, which is how its keys are read once for all of them.  A row whose
// keys lie in several units gets its pieces merged.
//
// bf16: as in the model's own attention, S^T = K Q^T on
// v_mfma_f32_32x32x16_bf16 puts one query's scores into one lane, and the K
// rows sit permuted in LDS so that a lane's scores are the 8 consecutive keys
// its operand of O^T += V^T P^T wants.  What differs:
//   * pages hold V row-major (one token is one contiguous write, a page copy
//     is one run), so its operand is formed by the transposing LDS read;
//   * tiles come through the page table: a 16-place group lies in one page, so
//     the DMA of 8 rows has a wave-uniform 64-bit base.  A wave keeps 64 table
//     entries in a register and reads them by lane;
//   * places outside the unit's keys are not read: their lanes fetch the
//     nearest valid place, and the scores are masked.  (An infinite value of
//     that place, times a probability of 0, is NaN where infinity was due.)
// Two kernels: branch_wide_kernel, 256 rows that share every tile (bound by the
// matrix cores and the softmax's arithmetic), and branch_few_kernel, up to 64
// rows whose keys are dealt to four waves (bound by reading the keys).  float32
// has branch_f32_kernel, of the second kind.
#include "xc_pool.h"

#include "xc_internal.h"

#include <math.h>

namespace xc {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;

// MFMA row R of a 32-key half tile -> key offset within the 64-key tile
__device__ __forceinline__ int key_of_row(int mt, int R) {
  const int g = R >> 3, hh = (R >> 2) & 1, r = R & 3;
  return mt * 32 + (g >> 1) * 16 + hh * 8 + (g & 1) * 4 + r;
}

// 16 bytes per lane, global -> LDS (lane l at byte 16 l of the wave's 1 KB
// block) from byte off past a wave-uniform base; a buffer load, so that LDS
// reads stay counted behind it
__device__ __forceinline__ void dma16(const char* base, unsigned off, char* lds_block) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), (short)0, -1, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds_block, 16, (int)off, 0, 0, 0);
}

// s_waitcnt vmcnt(n), the other counters left alone
#define XC_WAIT_VM(n) __builtin_amdgcn_s_waitcnt(0x0f70 | ((n) & 15) | (((n) >> 4) << 14))

__device__ __forceinline__ void tile_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ float partner_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float partner_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Where a query row's results go.
struct RowOut {
  long long out, piece, stat;
};
__device__ __forceinline__ RowOut row_out(const AttnArgs& a, const AttnUnit& un, int h, int r) {
  const int t = un.tok0 + r / a.group, qh = h * a.group + r % a.group;
  RowOut o;
  o.out = (long long)t * a.out_ld + qh * a.buf.D;
  o.stat = ((long long)un.slot * a.piece_rows + t - a.piece_row0) * a.q_heads + qh;
  o.piece = o.stat * a.buf.D;
  return o;
}

// The page table of a unit, 64 entries at a time: entry e0 + lane.
struct TableWindow {
  const int* table;
  int e0, e_last, entries, shift, lane;
  __device__ __forceinline__ TableWindow(const AttnArgs& a, const AttnUnit& un, int ln)
      : table(a.tables + un.table), e0(un.lo >> a.buf.shift), e_last((un.hi - 1) >> a.buf.shift), shift(a.buf.shift), lane(ln) {
    entries = table[min(e0 + lane, e_last)];
  }
  // from place `from` on the window covers places up to `to`; the load is
  // waited for here, not where an entry is read
  __device__ __forceinline__ void cover(int from, int to) {
    if ((to >> shift) - e0 >= 64) {
      e0 = from >> shift;
      entries = table[min(e0 + lane, e_last)];
      asm volatile("" : "+v"(entries));
    }
  }
  // page of place at, the same in all lanes
  __device__ __forceinline__ long long page(int at) const {
    return __builtin_amdgcn_readlane(entries, __builtin_amdgcn_readfirstlane(at >> shift) - e0);
  }
};

// Rows of 8 sixteen-byte chunks in LDS, 1 KB blocks of 8 rows; 8 lanes of a
// request fetch 128 contiguous bytes.  K: row r, chunk c at (r % 8 ^ r / 8 % 2)
// * 8 + (c ^ r % 8): the 16 rows that a quarter wave reads at one chunk fall
// into 16 bank groups.  V: r % 8 * 8 + (c ^ r / 2 % 2 * 4): so do the 4 rows x 4
// chunks that half a wave of a transposing read takes.  KCG blocks per 8 rows
// of D columns.
template <int D>
struct Frags {
  static constexpr int KCG = D / 64, DT = D / 32, KS = D / 16;
  int k_off[4], v_off[2];
  __device__ __forceinline__ explicit Frags(int lane) {
    const int hi = lane >> 5, lo = lane & 31;
    const int row = (lane >> 2) & 3;  // of a transposing read
#pragma unroll
    for (int i = 0; i < 4; ++i)
      k_off[i] = (lo >> 3) * KCG * 1024 + ((lo & 7) ^ ((lo >> 3) & 1)) * 128 + ((2 * i + hi) ^ (lo & 7)) * 16;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      v_off[i] = hi * KCG * 1024 + row * 128 + (i ^ (row >> 1)) * 64 + (((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) * 16 +
                 (lane & 1) * 8;
  }
  // keys of half tile mt, head dims ks * 16 + hi * 8 ..
  __device__ __forceinline__ bf16x8 k(const char* tile, int mt, int ks) const {
    return *reinterpret_cast<const bf16x8*>(tile + k_off[ks & 3] + mt * 4 * KCG * 1024 + (ks >> 2) * 1024);
  }
  // head dim dt * 32 + lo, keys kv * 16 + hi * 8 ..
  __device__ __forceinline__ bf16x8 v(const char* tile, int kv, int dt) const {
    const char* p = tile + v_off[dt & 1] + kv * 2 * KCG * 1024 + (dt >> 1) * 1024;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 512));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// A block's row and column bytes that lane `lane` fetches: block (rg, cg) of a
// K or a V tile.
__device__ __forceinline__ int k_block_row(int rg, int lane) {
  const int R = rg * 8 + ((lane >> 3) ^ (rg & 1));
  return key_of_row(R >> 5, R & 31);
}
__device__ __forceinline__ unsigned k_block_col(int rg, int cg, int lane) { return (cg * 8 + ((lane & 7) ^ (lane >> 3) ^ (rg & 1))) * 16; }
__device__ __forceinline__ int v_block_row(int rg, int lane) { return rg * 8 + (lane >> 3); }
__device__ __forceinline__ unsigned v_block_col(int cg, int lane) { return (cg * 8 + ((lane & 7) ^ (((lane >> 4) & 1) << 2))) * 16; }

// The address of a unit's query row r, head dims hi * 8 on.
__device__ __forceinline__ const bf16* query_row(const AttnArgs& a, const AttnUnit& un, int h, int r, int hi) {
  return reinterpret_cast<const bf16*>(a.q) + (un.tok0 + r / a.group) * a.q_ld +
         (long long)(h * a.group + r % a.group) * a.buf.D + hi * 8;
}

// Scores of keys outside [lo, last]: -infinity.  at0: the place of the half tile's first key.
__device__ __forceinline__ void mask_half(f32x16& s, int at0, int hi, int lo, int last) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int at = at0 + key_of_row(0, (i >> 2) * 8 + hi * 4 + (i & 3));
    if (at < lo || at > last) s[i] = -INFINITY;
  }
}
__device__ __forceinline__ float half_max(const f32x16& s) {
  float m = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
  return m;
}

// p = 2^(scale s - m), rounded to bf16 for the matrix cores (2^-8 each, of
// either sign); the sum takes them before that rounding (but see ONES below).
__device__ __forceinline__ float half_probs(const f32x16& s, float scale, float m, bf16x8 (&p)[2]) {
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale, -m));
    sum[i & 3] += e;
    p[i >> 3][i & 7] = (bf16)e;
  }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// The maximum before any key: a finite number, so that a score of -infinity (an
// overflowing product) is a probability of 0 beside it and not NaN.
constexpr float kNoMax = -3.402823466e38f;

// The maximum that exponents are taken against moves only when a tile's
// maximum exceeds it by more than this: p stays <= 2^8 in between.  The wide
// kernel looks at what the exponentials gave instead (see there): p stays below
// 2^13 at d = 128 and 2^9 at d = 64.  Float sums and bf16 carry any of them.
constexpr float kMaxSlack = 8.0f, kMaxP = 256.0f;

// 8 waves of 32 rows, all on the same tiles of 64 keys, two waves per SIMD in
// alternation: while one is on the matrix cores (S of the next tile and O of
// this one, a run of MFMAs and LDS reads), the other takes its softmax
// (vector instructions alone) and requests tiles; a barrier swaps them.  So
// both pipes have work at any time without any interleaving within a wave, and
// a wave needs one score tile instead of two.
//
// K and V rings of four slots.  Tile j + 3 is requested between the products
// of tile j, where the wave has issue slots to spare, and has landed three
// phases later at the earliest it may be read; the slot it goes to was last
// read by tile j - 1.
//
// Bound by the two phases: at d = 128 about 1150 cycles of softmax and 1430 of
// products, at d = 64 about 940 and 900, where the products alone are 1024
// and 640; a clock of 1.5 to 1.8 GHz is what the chip's power leaves with all
// CUs at it.  28080 rows, 21060 keys, 12 heads of 128: 2.99 to 3.13 ms from
// card to card, 1160 to 1210 TFLOP/s; 6144 rows, 2304 keys, 8 heads of 64: 40 us, 720 TFLOP/s.  The former with
// other choices, at 3440 or 3330 us before the last round of workgroups was
// filled: the matrix phase without a raised wave priority 3760 us
// instead of 3440, the softmax raised instead 4010; the softmax not held before
// its barrier 3800; a maximum per tile 3440 instead of 3330 (51 us instead of 45
// for the latter).  One wave of 64 rows per SIMD, its softmax between its own
// products, halves the LDS reads but has nothing to hide the requests' address
// arithmetic behind: 3650 instead of 3310 (47 instead of 43).
template <int D>
__global__ __launch_bounds__(64 * kWaves, 1) void branch_wide_kernel(AttnArgs a) {
  using F = Frags<D>;
  constexpr int KCG = F::KCG, DT = F::DT, KS = F::KS;
  constexpr int NB = 8 * KCG / kWaves;  // blocks per wave, of a K or a V tile
  // d = 64, where the softmax is the longer phase: its row sums are products
  // with a row of ones, and so sums (in float) of the rounded probabilities: 2^-8
  // more of the result at worst, but the numerator's own roundings where all go
  // one way cancel
  constexpr int ONES = D == 64;
  constexpr int SLOT = 64 * D * 2;
  // an array per slot: its reads then do not wait for requests into the others
  // (K's come after V's in LDS, in order of name: a transposing read's offset
  // folds into the instruction only below 64 KB)
  __shared__ __attribute__((aligned(1024))) char tK0[SLOT];
  __shared__ __attribute__((aligned(1024))) char tK1[SLOT];
  __shared__ __attribute__((aligned(1024))) char tK2[SLOT];
  __shared__ __attribute__((aligned(1024))) char tK3[SLOT];
  __shared__ __attribute__((aligned(1024))) char sV0[SLOT];
  __shared__ __attribute__((aligned(1024))) char sV1[SLOT];
  __shared__ __attribute__((aligned(1024))) char sV2[SLOT];
  __shared__ __attribute__((aligned(1024))) char sV3[SLOT];
  int u, h;
  if (!xcd_pair(blockIdx.x, a.n_units, a.n_long, a.buf.kv_heads, u, h)) return;
  const AttnUnit un = a.units[u];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const int rows = un.tokens * a.group;
  const int base = un.lo & ~15, n = (un.hi - base + 63) >> 6, last = un.hi - 1;
  const bool live = wave * 32 < rows, later = wave >= kWaves / 2;
  const int in_page = (1 << a.buf.shift) - 1;
  const long long head_bytes = (long long)D * 2 << a.buf.shift, page_bytes = head_bytes * a.buf.kv_heads;
  const char* Kh = reinterpret_cast<const char*>(a.buf.keys) + h * head_bytes;
  const char* Vh = reinterpret_cast<const char*>(a.buf.values) + h * head_bytes;
  TableWindow win(a, un, lane);

  // Block i of this wave: rows 8 rg .. of the tile, all in the 16-place group
  // rg / 2.  Past the last key its row is read instead (the scores are masked),
  // past the last tile that tile: the number of requests in flight is then
  // always the same, and waits can count them.
  int k_row[NB], v_row[NB];
  unsigned k_col[NB], v_col[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int B = wave + kWaves * i, rg = B / KCG, cg = B % KCG;
    k_row[i] = k_block_row(rg, lane) & 15;
    k_col[i] = k_block_col(rg, cg, lane);
    v_row[i] = v_block_row(rg, lane) & 15;
    v_col[i] = v_block_col(cg, lane);
  }
  const unsigned page_kb = (unsigned)(page_bytes >> 10);
  long long group_at = 0;  // of block i of the tile being requested: bytes of its 16-place group
  int group_rows = 15;
  // half a request: K (first) or V of block i of tile j; j0: the unit's first tile
  auto fetch = [&](int j, int i, bool is_v, char* dst, bool j0 = false) __attribute__((always_inline)) {
    if (!is_v) {
      const int g0 = min(base + min(j, n - 1) * 64 + (wave + kWaves * i) / KCG / 2 * 16, last & ~15);
      const int page = __builtin_amdgcn_readlane(win.entries, (g0 >> a.buf.shift) - win.e0);
      group_at = ((long long)((unsigned)page * page_kb) << 10) + (g0 & in_page) * (D * 2);
      group_rows = min(15, last - g0);
    }
    if (dst == nullptr) return;  // only the address
    int row = min(is_v ? v_row[i] : k_row[i], group_rows);
    if (j0) row = max(row, un.lo - base - (wave + kWaves * i) / KCG / 2 * 16);
    dma16((is_v ? Vh : Kh) + group_at, row * (D * 2) + (is_v ? v_col[i] : k_col[i]), dst + (wave + kWaves * i) * 1024);
  };
  auto cover = [&](int j) __attribute__((always_inline)) {
    const int at0 = base + min(j, n - 1) * 64;
    win.cover(max(at0, un.lo), min(at0 + 63, last));
  };
  auto request = [&](int j, char* kd, char* vd, bool j0 = false) __attribute__((always_inline)) {
    cover(j);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      fetch(j, i, false, kd, j0);
      fetch(j, i, true, vd, j0);
    }
  };
  // What S of the first tile needs is asked for first and waited for alone (36
  // tiles, d = 128: 64 us instead of 65).
#pragma unroll
  for (int i = 0; i < NB; ++i) fetch(0, i, false, tK0, true);
  bf16x8 qf[KS];
  if (live) {
    const bf16* q = query_row(a, un, h, min(wave * 32 + lo, rows - 1), hi);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(q + ks * 16);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    fetch(0, i, false, nullptr, true);
    fetch(0, i, true, sV0, true);
  }
  request(1, tK1, sV1);
  request(2, tK2, sV2);
  if (!live) {
    // waves without rows only stage tiles, between the same barriers
    XC_WAIT_VM(0);
    tile_barrier();
    tile_barrier();
    if (later) tile_barrier();
    auto stage = [&](int j, char* kd, char* vd) __attribute__((always_inline)) {
      if (!later) XC_WAIT_VM(2 * NB);
      tile_barrier();
      request(j + 3, kd, vd);
      if (later) XC_WAIT_VM(2 * NB);
      tile_barrier();
    };
    for (int j = 0; j < n - 1; j += 4) {
      stage(j, tK3, sV3);
      if (j + 1 >= n - 1) break;
      stage(j + 1, tK0, sV0);
      if (j + 2 >= n - 1) break;
      stage(j + 2, tK1, sV1);
      if (j + 3 >= n - 1) break;
      stage(j + 3, tK2, sV2);
    }
    if (!later) tile_barrier();
    return;
  }

  f32x16 s[2], oacc[DT + ONES];
#pragma unroll
  for (int i = 0; i < DT + ONES; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  float m_run = kNoMax, l_run = 0.f;
  bf16x8 p[2][2], ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (bf16)1.0f;
  const F f(lane);
  // The matrix phase as a fixed sequence: 4 (DT + ONES) products P V, then 2 KS
  // products K Q^T, one fragment each, read PF products ahead (an LDS read
  // takes longer than the one product that the compiler would read ahead).
  constexpr int PF = 4, NPV = 4 * (DT + ONES), NQK = 2 * KS;
  bf16x8 fr[PF];
  auto frag = [&](int i, const char* vt, const char* kt) __attribute__((always_inline)) {
    if (i >= NPV) return f.k(kt, (i - NPV) & 1, (i - NPV) >> 1);
    return i % (DT + ONES) < DT ? f.v(vt, i / (DT + ONES), i % (DT + ONES)) : ones;
  };
  auto product = [&](int i, const bf16x8& x) __attribute__((always_inline)) {
    if (i < NPV) {
      const int kv = i / (DT + ONES), dt = i % (DT + ONES);
      oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[kv >> 1][kv & 1], oacc[dt], 0, 0, 0);
    } else {
      const int mt = (i - NPV) & 1, ks = (i - NPV) >> 1;
      if (ks == 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[mt][r] = 0.f;
      }
      s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[ks], s[mt], 0, 0, 0);
    }
  };
  // products [i0, i1); the first PF fragments are in fr; aside(i) goes between them
  auto products = [&](int i0, int i1, const char* vt, const char* kt, auto&& aside) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NPV + NQK; ++i) {
      if (i < i0 || i >= i1) continue;
      const bf16x8 x = fr[i % PF];
      if (i + PF < i1) fr[i % PF] = frag(i + PF, vt, kt);
      product(i, x);
      aside(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto nothing = [](int) __attribute__((always_inline)) {};
  auto lead = [&](int i0, const char* vt, const char* kt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PF; ++i) fr[(i0 + i) % PF] = frag(i0 + i, vt, kt);
  };
  // Probabilities of the tile against the maximum so far, which is looked for
  // only where they grew (from the first tile's maximum) - most tiles need none.
  // Then the tile's own maximum joins in and everything so far is rescaled.  The
  // limit is checked on a lane's sum of 32, 2^kMaxSlack each (one of them may reach
  // 2^13), or, where there is none, on the bf16 exponents, whose highest bit
  // stands for 2 and more: the maximum is taken kMaxSlack higher there (2^9 above it).
  float l_tile = 0.f;
  auto exps = [&]() __attribute__((always_inline)) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][i], a.scale, -m_run));
        if (!ONES) sum[i & 3] += e;
        p[mt][i >> 3][i & 7] = (bf16)e;
      }
    if (!ONES) {
      const float t = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      l_tile = t;
      return !(t <= 32.f * kMaxP);
    }
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    u32x4 b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = __builtin_bit_cast(u32x4, p[k >> 1][k & 1]);
    const u32x4 o = (b[0] | b[1]) | (b[2] | b[3]);
    return (((o[0] | o[1]) | (o[2] | o[3])) & 0x40004000u) != 0;
  };
  auto softmax = [&]() __attribute__((always_inline)) {
    const bool grew = exps();
    if (__builtin_amdgcn_ballot_w64(grew) != 0) {
      const float mx = partner_max(fmaxf(half_max(s[0]), half_max(s[1]))) * a.scale + (ONES ? kMaxSlack : 0.f);
      const float m_new = fmaxf(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT + ONES; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
      m_run = m_new;
      exps();
    }
    if (!ONES) l_run += l_tile;
  };
  // only a unit's first and last tiles reach outside its keys
  auto mask = [&](int j) __attribute__((always_inline)) {
    mask_half(s[0], base + j * 64, hi, un.lo, last);
    mask_half(s[1], base + j * 64 + 32, hi, un.lo, last);
  };

  XC_WAIT_VM(5 * NB);  // the first K, the queries
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
  tile_barrier();
  lead(NPV, sV0, tK0);
  products(NPV, NPV + NQK, sV0, tK0, nothing);
  if (un.lo != base && n > 1) mask(0);
  // (keys that are yet to be masked are copies of valid ones)
  m_run = fmaxf(kNoMax, partner_max(fmaxf(half_max(s[0]), half_max(s[1]))) * a.scale + (ONES ? kMaxSlack : 0.f));
  XC_WAIT_VM(4 * NB);  // the first V
  tile_barrier();
  if (later) {
    XC_WAIT_VM(2 * NB);  // the second tile
    tile_barrier();
  }
  // tile j: its V, the next K, and the slots of tile j + 3
  auto iter = [&](int j, const char* vt, const char* kn, char* kd, char* vd) __attribute__((always_inline)) {
    softmax();
    // ... all of it here: without this the compiler sinks it behind the barrier, to P's use
    asm volatile("" : "+v"(p[0][0]), "+v"(p[0][1]), "+v"(p[1][0]), "+v"(p[1][1]), "+v"(l_run));
    lead(0, vt, kn);  // V has been there for a phase at least
    if (!later) XC_WAIT_VM(2 * NB);  // all but tile j + 2
    tile_barrier();
    cover(j + 3);
    __builtin_amdgcn_s_setprio(1);
    products(0, NPV + NQK, vt, kn, [&](int i) __attribute__((always_inline)) {
      constexpr int GAP = (NPV + NQK) / (2 * NB);
      if (i % GAP == 1) fetch(j + 3, i / GAP / 2, (i / GAP & 1) != 0, i / GAP & 1 ? vd : kd);
    });
    __builtin_amdgcn_s_setprio(0);
    if (later) XC_WAIT_VM(2 * NB);  // all but tile j + 3
    tile_barrier();
  };
  for (int j = 0; j < n - 1; j += 4) {
    iter(j, sV0, tK1, tK3, sV3);
    if (j + 1 >= n - 1) break;
    iter(j + 1, sV1, tK2, tK0, sV0);
    if (j + 2 >= n - 1) break;
    iter(j + 2, sV2, tK3, tK1, sV1);
    if (j + 3 >= n - 1) break;
    iter(j + 3, sV3, tK0, tK2, sV2);
  }
  if (!later) tile_barrier();
  {
    const int slot = (n - 1) & 3;
    const char* vt = slot == 0 ? sV0 : slot == 1 ? sV1 : slot == 2 ? sV2 : sV3;
    mask(n - 1);
    softmax();
    lead(0, vt, nullptr);
    products(0, NPV, vt, nullptr, nothing);
  }
  const int r = wave * 32 + lo;
  const float l = ONES ? oacc[DT][0] : partner_sum(l_run);
  if (r >= rows) return;
  const RowOut o = row_out(a, un, h, r);
  if (un.slot < 0) {
    const float inv = 1.0f / l;
    bf16* row = reinterpret_cast<bf16*>(a.out) + o.out;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (bf16)(oacc[dt][g * 4 + i] * inv);
        *reinterpret_cast<bf16x4*>(row + dt * 32 + g * 8 + hi * 4) = v;
      }
  } else {
    float* row = a.pieces + o.piece;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = oacc[dt][g * 4 + i];
        *reinterpret_cast<f32x4*>(row + dt * 32 + g * 8 + hi * 4) = v;
      }
    if (hi == 0) a.stats[o.stat] = make_float2(m_run, l);
  }
}

// Up to 64 rows: four waves, each with all rows (G groups of 32) on keys of
// its own: tiles of 32 keys (64 at d = 64), dealt in turn.  A wave has a K and a V
// tile of its own in LDS, asks for the next K as soon as S is formed and for the
// next V after P V, and waits for nothing but its own requests; there is no
// barrier until the four partial results are joined in LDS at the end.  80 KB
// of LDS: two workgroups, eight waves per CU, 128 KB in flight.  Two groups read
// their queries from LDS in every tile: with two output accumulators there
// are no registers for them.
//
// Bound by reading keys and values: 16 rows over 14200 keys, 12 heads of 128
// (101 MB) 25.6 us with the merge, 64 rows over 36600 keys, 16 heads of 128
// (658 MB) 120 us (141 as two workgroups of one row group each, before requests
// fetched whole 128-byte lines), 64 rows over 2000 keys of their own, 16 heads of
// 128 (1049 MB) 172 us, 6.1 TB/s.
template <int D>
struct FewShape {
  static constexpr int HT = 128 / D;                  // 32-key halves of a tile
  static constexpr int KEYS = 32 * HT;
  static constexpr int TILE = KEYS * D * 2;           // bytes, 8 KB
  static constexpr int LOADS = TILE / 1024;
};
template <int D, int G>
__device__ __forceinline__ void few_body(const AttnArgs& a, const AttnUnit& un, int h, char* sK, char* sV, char* sQ) {
  using F = Frags<D>;
  using S = FewShape<D>;
  constexpr int KCG = F::KCG, DT = F::DT, KS = F::KS, HT = S::HT;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const int rows = un.tokens * a.group;
  const int base = un.lo & ~15, last = un.hi - 1;
  const int tiles = (un.hi - base + S::KEYS - 1) / S::KEYS;
  const int n = (tiles - wave + 3) >> 2;  // this wave's: wave, wave + 4, ..
  const int in_page = (1 << a.buf.shift) - 1;
  const long long head_bytes = (long long)D * 2 << a.buf.shift, page_bytes = head_bytes * a.buf.kv_heads;
  const char* Kh = reinterpret_cast<const char*>(a.buf.keys) + h * head_bytes;
  const char* Vh = reinterpret_cast<const char*>(a.buf.values) + h * head_bytes;
  TableWindow win(a, un, lane);
  // the queries are asked for first and waited for before the loop, which
  // would otherwise drain the requests behind them in every tile
  bf16x8 qf[KS];
  if (G == 1) {
    const bf16* q = query_row(a, un, h, min(lo, rows - 1), hi);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(q + ks * 16);
  } else {
    // fragment (g, ks) as 64 lanes of 16 bytes; a wave brings in a quarter
#pragma unroll
    for (int i = 0; i < G * KS / 4; ++i) {
      const int fi = wave * (G * KS / 4) + i, g = fi / KS, ks = fi % KS;
      const bf16x8 q = *reinterpret_cast<const bf16x8*>(query_row(a, un, h, min(g * 32 + lo, rows - 1), hi) + ks * 16);
      *reinterpret_cast<bf16x8*>(sQ + fi * 1024 + lane * 16) = q;
    }
  }
  char* kt = sK + wave * S::TILE;
  char* vt = sV + wave * S::TILE;
  // tile i of this wave, of K (is_k) or V
  auto request = [&](int i, bool is_k) __attribute__((always_inline)) {
    const int at0 = base + (wave + 4 * i) * S::KEYS;
#pragma unroll
    for (int rg = 0; rg < 4 * HT; ++rg) {
      const int at = min(max(at0 + (is_k ? k_block_row(rg, lane) : v_block_row(rg, lane)), un.lo), last);
      const char* src = (is_k ? Kh : Vh) + win.page(min(max(at0 + (rg >> 1) * 16, un.lo), last)) * page_bytes;
#pragma unroll
      for (int cg = 0; cg < KCG; ++cg)
        dma16(src, (unsigned)(at & in_page) * (D * 2) + (is_k ? k_block_col(rg, cg, lane) : v_block_col(cg, lane)),
              (is_k ? kt : vt) + (rg * KCG + cg) * 1024);
    }
  };
  auto cover = [&](int i) __attribute__((always_inline)) {
    const int at0 = base + (wave + 4 * i) * S::KEYS;
    win.cover(max(at0, un.lo), min(at0 + S::KEYS - 1, last));
  };
  if (n > 0) {
    cover(0);
    request(0, true);
    request(0, false);
  }
  if (G == 1) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
  } else {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    tile_barrier();
  }
  f32x16 oacc[G][DT];
  float m_run[G], l_run[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    m_run[g] = kNoMax;
    l_run[g] = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[g][i][r] = 0.f;
  }
  const F f(lane);
  for (int i = 0; i < n; ++i) {
    XC_WAIT_VM(S::LOADS);  // K has landed, V may be on its way
    asm volatile("" ::: "memory");
    f32x16 s[G][HT];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int mt = 0; mt < HT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[g][mt][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 q[G];
#pragma unroll
      for (int g = 0; g < G; ++g)
        q[g] = G == 1 ? qf[ks] : *reinterpret_cast<const bf16x8*>(sQ + (g * KS + ks) * 1024 + lane * 16);
#pragma unroll
      for (int mt = 0; mt < HT; ++mt) {
        const bf16x8 k = f.k(kt, mt, ks);
#pragma unroll
        for (int g = 0; g < G; ++g) s[g][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[g], s[g][mt], 0, 0, 0);
      }
    }
    const bool more = i + 1 < n;
    if (more) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this K has been read
      cover(i + 1);
      request(i + 1, true);
    }
    const int tile = wave + 4 * i;
    bf16x8 p[G][HT][2];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (tile == 0 || tile == tiles - 1) {
#pragma unroll
        for (int mt = 0; mt < HT; ++mt) mask_half(s[g][mt], base + tile * S::KEYS + mt * 32, hi, un.lo, last);
      }
      float mx = half_max(s[g][0]);
#pragma unroll
      for (int mt = 1; mt < HT; ++mt) mx = fmaxf(mx, half_max(s[g][mt]));
      mx = partner_max(mx) * a.scale;
      if (mx > m_run[g] + kMaxSlack) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[g] - mx);
        l_run[g] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[g][dt][r] *= alpha;
        m_run[g] = mx;
      }
#pragma unroll
      for (int mt = 0; mt < HT; ++mt) l_run[g] += half_probs(s[g][mt], a.scale, m_run[g], p[g][mt]);
    }
    if (more) { XC_WAIT_VM(S::LOADS); } else { XC_WAIT_VM(0); }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int kv = 0; kv < 2 * HT; ++kv)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 v = f.v(vt, kv, dt);
#pragma unroll
        for (int g = 0; g < G; ++g)
          oacc[g][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[g][kv >> 1][kv & 1], oacc[g][dt], 0, 0, 0);
      }
    if (more) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this V has been read
      request(i + 1, false);
    }
  }

  // Join the four waves' results, one group of rows after the other: (max, sum)
  // in the queries' place and unnormalised outputs, waves 0 and 1 in the K
  // tiles, 2 and 3 in the V tiles; chunk c of row r sits at c ^ r, so that
  // lanes with different rows meet different banks.
  constexpr int LPR = D / 4;  // 16-byte chunks, or lanes, per row
  static_assert(2 * 32 * D * 4 <= 4 * S::TILE, "two partial results per array");
  float2* stats = reinterpret_cast<float2*>(sQ);
  auto part = [&](int w, int r, int c) __attribute__((always_inline)) {
    return reinterpret_cast<f32x4*>(w < 2 ? sK : sV) + ((w & 1) * 32 + r) * LPR + (c ^ (r & (LPR - 1)));
  };
#pragma unroll
  for (int g = 0; g < G; ++g) {
    __syncthreads();
    {
      const float l = partner_sum(l_run[g]);
      if (hi == 0) stats[wave * 32 + lo] = make_float2(m_run[g], l);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x4 v;
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = oacc[g][dt][e * 4 + k];
          *part(wave, lo, dt * 8 + e * 2 + hi) = v;
        }
    }
    __syncthreads();
    const int c = tid % LPR;
    for (int r = tid / LPR; r < min(32, rows - g * 32); r += 256 / LPR) {
      float m = stats[r].x, l = 0.f;
#pragma unroll
      for (int k = 1; k < 4; ++k) m = fmaxf(m, stats[k * 32 + r].x);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 st = stats[k * 32 + r];
        const float w = k < tiles ? __builtin_amdgcn_exp2f(st.x - m) : 0.f;  // a wave without tiles adds nothing
        l += w * st.y;
        o += w * *part(k, r, c);
      }
      const RowOut ro = row_out(a, un, h, g * 32 + r);
      if (un.slot < 0) {
        const float inv = 1.0f / l;
        bf16x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (bf16)(o[k] * inv);
        *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16*>(a.out) + ro.out + c * 4) = v;
      } else {
        *reinterpret_cast<f32x4*>(a.pieces + ro.piece + c * 4) = o;
        if (c == 0) a.stats[ro.stat] = make_float2(m, l);
      }
    }
  }
}
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void branch_few_kernel(AttnArgs a) {
  // arrays of their own: reads of one then do not wait for requests into another
  __shared__ __attribute__((aligned(1024))) char sK[4 * FewShape<D>::TILE];
  __shared__ __attribute__((aligned(1024))) char sV[4 * FewShape<D>::TILE];
  __shared__ __attribute__((aligned(1024))) char sQ[64 * D * 2];
  // units outermost, the long ones first: each key is read by one workgroup
  // (or two in a row), so what counts is that the CUs finish together
  const int u = blockIdx.x / a.buf.kv_heads, h = blockIdx.x - u * a.buf.kv_heads;
  const AttnUnit un = a.units[u];
  if (un.tokens * a.group > 32) few_body<D, 2>(a, un, h, sK, sV, sQ);
  else few_body<D, 1>(a, un, h, sK, sV, sQ);
}

// float32: as branch_few_kernel, four waves with all of up to 32 rows on 32-key
// tiles of their own, on v_mfma_f32_32x32x2_f32.  The two k indices of a product
// are any two head dims (S) or keys (P V) as long as both operands agree, so
// no operand needs a shuffle: S takes dims 8 t + e and 8 t + 4 + e, P V the two
// keys whose scores sit in one register of the two half-waves.  Bound by these
// products (64 cycles each).  Many rows are dealt to more workgroups: four waves
// of 32 rows on shared tiles, staged through registers, took 456 us for 2000
// rows, 4500 keys, 8 heads of 128, where these took 388 (350 now, 105
// TFLOP/s: the matrix units are busy 70% of the cycles), and 9.9 us for the tiny
// model's 3 x 64 rows and 128 keys, where these take 5.1.
// Row r, chunk c of a tile sits at c ^ f(r): rows at one chunk (K) and one row's
// chunks beside those of the row 4 below (V) meet different banks.
template <int D>
__global__ __launch_bounds__(256, 1) void branch_f32_kernel(AttnArgs a) {
  constexpr int DT = D / 32, CH = D / 4, TILE = 32 * D * 4, LOADS = TILE / 1024, RPB = 64 / CH;  // rows per 1 KB block
  __shared__ __attribute__((aligned(1024))) char sK[4 * TILE];
  __shared__ __attribute__((aligned(1024))) char sV[4 * TILE];
  __shared__ float2 stats[4][32];
  const int u = blockIdx.x / a.buf.kv_heads, h = blockIdx.x - u * a.buf.kv_heads;
  const AttnUnit un = a.units[u];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const int rows = un.tokens * a.group;
  const int base = un.lo & ~15, last = un.hi - 1;
  const int tiles = (un.hi - base + 31) >> 5;
  const int n = (tiles - wave + 3) >> 2;
  const int in_page = (1 << a.buf.shift) - 1;
  const long long head_bytes = (long long)D * 4 << a.buf.shift, page_bytes = head_bytes * a.buf.kv_heads;
  const char* Kh = reinterpret_cast<const char*>(a.buf.keys) + h * head_bytes;
  const char* Vh = reinterpret_cast<const char*>(a.buf.values) + h * head_bytes;
  TableWindow win(a, un, lane);
  char* kt = sK + wave * TILE;
  char* vt = sV + wave * TILE;
  auto swz = [](int r, int c) __attribute__((always_inline)) {
    return c ^ (CH >= 16 ? (r & 7) ^ ((r & 4) << 1) : r & 7);
  };
  auto request = [&](int i, const char* src, char* dst) __attribute__((always_inline)) {
    const int at0 = base + (wave + 4 * i) * 32;
#pragma unroll
    for (int b = 0; b < LOADS; ++b) {
      const int row = b * RPB + lane / CH, g0 = at0 + (b * RPB & 16);
      const int at = min(max(at0 + row, un.lo), last);
      dma16(src + win.page(min(max(g0, un.lo), last)) * page_bytes,
            (unsigned)(at & in_page) * (D * 4) + swz(row, lane % CH) * 16, dst + b * 1024);
    }
  };
  auto cover = [&](int i) __attribute__((always_inline)) {
    const int at0 = base + (wave + 4 * i) * 32;
    win.cover(max(at0, un.lo), min(at0 + 31, last));
  };
  f32x4 qf[D / 8];
  {
    const int r = min(lo, rows - 1);
    const float* q = reinterpret_cast<const float*>(a.q) + (un.tok0 + r / a.group) * a.q_ld +
                     (long long)(h * a.group + r % a.group) * D + hi * 4;
#pragma unroll
    for (int t = 0; t < D / 8; ++t) qf[t] = *reinterpret_cast<const f32x4*>(q + t * 8);
  }
  if (n > 0) {
    cover(0);
    request(0, Kh, kt);
    request(0, Vh, vt);
  }
#pragma unroll
  for (int t = 0; t < D / 8; ++t) asm volatile("" : "+v"(qf[t]));
  f32x16 oacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  float m_run = kNoMax, l_run = 0.f;
  for (int i = 0; i < n; ++i) {
    XC_WAIT_VM(LOADS);  // K has landed, V may be on its way
    asm volatile("" ::: "memory");
    f32x16 s, s1;  // two sums: no product waits for the one before it
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = s1[r] = 0.f;
#pragma unroll
    for (int t = 0; t < D / 8; ++t) {
      const f32x4 k = *reinterpret_cast<const f32x4*>(kt + lo * (D * 4) + swz(lo, t * 2 + hi) * 16);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], qf[t][e], s, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e + 1], qf[t][e + 1], s1, 0, 0, 0);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] += s1[r];
    const bool more = i + 1 < n;
    if (more) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this K has been read
      cover(i + 1);
      request(i + 1, Kh, kt);
    }
    const int tile = wave + 4 * i;
    if (tile == 0 || tile == tiles - 1) {  // only these reach outside the unit's keys
      const int at0 = base + tile * 32;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int at = at0 + (r >> 2) * 8 + hi * 4 + (r & 3);
        if (at < un.lo || at > last) s[r] = -INFINITY;
      }
    }
    const float mx = partner_max(half_max(s)) * a.scale;
    if (mx > m_run + kMaxSlack) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
      m_run = mx;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale, -m_run));
      l_run += s[r];
    }
    if (more) { XC_WAIT_VM(LOADS); } else { XC_WAIT_VM(0); }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = (r >> 2) * 8 + hi * 4 + (r & 3);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const float v = *reinterpret_cast<const float*>(vt + key * (D * 4) + swz(key, dt * 8 + (lo >> 2)) * 16 + (lo & 3) * 4);
        oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[r], oacc[dt], 0, 0, 0);
      }
    }
    if (more) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this V has been read
      request(i + 1, Vh, vt);
    }
  }
  __syncthreads();
  auto part = [&](int w, int r, int c) __attribute__((always_inline)) {
    return reinterpret_cast<f32x4*>(sK + w * TILE) + r * CH + (c ^ (r & 7));
  };
  {
    const float l = partner_sum(l_run);
    if (hi == 0) stats[wave][lo] = make_float2(m_run, l);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = oacc[dt][e * 4 + k];
        *part(wave, lo, dt * 8 + e * 2 + hi) = v;
      }
  }
  __syncthreads();
  const int c = tid % CH;
  for (int r = tid / CH; r < rows; r += 256 / CH) {
    float m = stats[0][r].x, l = 0.f;
#pragma unroll
    for (int k = 1; k < 4; ++k) m = fmaxf(m, stats[k][r].x);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 st = stats[k][r];
      const float w = k < tiles ? exp2f(st.x - m) : 0.f;  // a wave without tiles adds nothing
      l += w * st.y;
      o += w * *part(k, r, c);
    }
    const RowOut ro = row_out(a, un, h, r);
    if (un.slot < 0) {
      const float inv = 1.0f / l;
      *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + ro.out + c * 4) = o * inv;
    } else {
      *reinterpret_cast<f32x4*>(a.pieces + ro.piece + c * 4) = o;
      if (c == 0) a.stats[ro.stat] = make_float2(m, l);
    }
  }
}

// Joins the pieces of each (row, query head):
// O = sum_p w_p O_p / sum_p w_p l_p, w_p = 2^(m_p - max m).
// A wave owns one of them.  It is a chain of memory latencies, so what is
// independent is in flight together: all statistics (a lane per piece) and
// the outputs, each of 64 / (D / 4) lane groups taking every so many pieces,
// eight at a time.  Every sum has a fixed order.  4 to 5 us for 192 rows of 15
// pieces and for 1024 of 13.
template <typename T, int D>
__global__ __launch_bounds__(256) void branch_merge_kernel(AttnArgs a) {
  constexpr int LPH = D / 4, NG = 64 / LPH, U = 8;
  const int lane = threadIdx.x & 63, g = lane / LPH, d0 = lane % LPH * 4;
  const long long i = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long rq = (long long)a.piece_rows * a.q_heads;
  if (i >= rq) return;
  const int t = a.piece_row0 + (int)(i / a.q_heads);
  const OwnSlots own = a.own[t];
  const int n = a.shared_slots + own.n;
  if (n == 0) return;  // written by its only unit
  auto slot = [&](int p) __attribute__((always_inline)) {
    return (long long)(p < a.shared_slots ? p : own.first + p - a.shared_slots) * rq + i;
  };
  static_assert(kPlanMaxSlots <= 128, "two pieces' statistics per lane");
  float2 st[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) st[k] = a.stats[slot(min(lane + 64 * k, n - 1))];
  f32x4 o[U];
  auto fetch = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int p = p0 + k * NG + g;
      if (p < n) o[k] = *reinterpret_cast<const f32x4*>(a.pieces + slot(p) * D + d0);
    }
  };
  fetch(0);
  float m = fmaxf(st[0].x, st[1].x);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  float w[2], den = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    w[k] = lane + 64 * k < n ? exp2f(st[k].x - m) : 0.f;
    den += w[k] * st[k].y;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) den += __shfl_xor(den, off, 64);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0;;) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int p = p0 + k * NG + g;
      const float w0 = __shfl(w[0], p & 63, 64), w1 = __shfl(w[1], p & 63, 64);
      if (p < n) acc += (p < 64 ? w0 : w1) * o[k];
    }
    p0 += NG * U;
    if (p0 >= n) break;
    fetch(p0);
  }
#pragma unroll
  for (int off = 32; off >= LPH; off >>= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], off, 64);
  if (g != 0) return;
  T* out = reinterpret_cast<T*>(a.out) + t * a.out_ld + (i % a.q_heads) * D + d0;
  const float inv = 1.0f / den;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (T)(acc[e] * inv);
}

// The same where at most kFewPieces pieces join: each group of D / 4 lanes owns
// a (row, query head), and everything it reads is in flight at once.
constexpr int kFewPieces = 6;
template <typename T, int D>
__global__ __launch_bounds__(256) void branch_merge_few_kernel(AttnArgs a) {
  constexpr int LPH = D / 4;
  const long long i = (long long)blockIdx.x * (256 / LPH) + threadIdx.x / LPH;
  const int d0 = threadIdx.x % LPH * 4;
  const long long rq = (long long)a.piece_rows * a.q_heads;
  if (i >= rq) return;
  const int t = a.piece_row0 + (int)(i / a.q_heads);
  const OwnSlots own = a.own[t];
  const int n = a.shared_slots + own.n;
  if (n == 0) return;  // written by its only unit
  float2 st[kFewPieces];
  f32x4 o[kFewPieces];
#pragma unroll
  for (int k = 0; k < kFewPieces; ++k) {
    const int p = min(k, n - 1);
    const long long at = (p < a.shared_slots ? p : own.first + p - a.shared_slots) * rq + i;
    if (k < a.n_slots) {
      st[k] = a.stats[at];
      o[k] = *reinterpret_cast<const f32x4*>(a.pieces + at * D + d0);
    }
  }
  float m = st[0].x, den = 0.f;
#pragma unroll
  for (int k = 1; k < kFewPieces; ++k)
    if (k < n) m = fmaxf(m, st[k].x);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kFewPieces; ++k)
    if (k < n) {
      const float w = exp2f(st[k].x - m);
      den += w * st[k].y;
      acc += w * o[k];
    }
  const float inv = 1.0f / den;
  typedef T vec __attribute__((ext_vector_type(4)));
  vec v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (T)(acc[e] * inv);
  *reinterpret_cast<vec*>(reinterpret_cast<T*>(a.out) + t * a.out_ld + (i % a.q_heads) * D + d0) = v;
}

}  // namespace

// Requirements (the caller's): D in {64, 128} (float32: 32 too); every unit
// has at least one key and at most kWideRows query rows (few: kFewRows,
// float32: kF32Rows); page tables, slots and piece buffers cover what the units name.
hipError_t launch_branch_attention(int dtype, const AttnArgs& a, hipStream_t st) {
  const int total = a.n_units * a.buf.kv_heads, D = a.buf.D;
  if (total == 0) return hipSuccess;
  const unsigned grid = (unsigned)xcd_grid(a.n_units, a.buf.kv_heads);
  if (dtype == 1) {
    if (a.few) {
      if (D == 128) branch_few_kernel<128><<<total, 256, 0, st>>>(a);
      else branch_few_kernel<64><<<total, 256, 0, st>>>(a);
    } else {
      if (D == 128) branch_wide_kernel<128><<<grid, 64 * kWaves, 0, st>>>(a);
      else branch_wide_kernel<64><<<grid, 64 * kWaves, 0, st>>>(a);
    }
  } else {
    if (D == 128) branch_f32_kernel<128><<<total, 256, 0, st>>>(a);
    else if (D == 64) branch_f32_kernel<64><<<total, 256, 0, st>>>(a);
    else branch_f32_kernel<32><<<total, 256, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_slots == 0) return e;
  // a wave per (row, head), or one of its lane groups where few pieces join.
  // 18096 of them with 3 pieces, d = 64: 48.3 us for the call, 50.7 with a wave
  // each; 1024 with 13 pieces need a wave each (no group could hold them).
  const bool few_pieces = a.n_slots <= kFewPieces;
  const long long rq = (long long)a.piece_rows * a.q_heads, per = few_pieces ? 256 / (D / 4) : 4;
  const unsigned mg = (unsigned)((rq + per - 1) / per);
#define XC_MERGE(T, DD)                                                     \
  do {                                                                      \
    if (few_pieces) branch_merge_few_kernel<T, DD><<<mg, 256, 0, st>>>(a);  \
    else branch_merge_kernel<T, DD><<<mg, 256, 0, st>>>(a);                 \
  } while (0)
  if (dtype == 1) {
    if (D == 128) XC_MERGE(bf16, 128);
    else XC_MERGE(bf16, 64);
  } else {
    if (D == 128) XC_MERGE(float, 128);
    else if (D == 64) XC_MERGE(float, 64);
    else XC_MERGE(float, 32);
  }
#undef XC_MERGE
  return hipGetLastError();
}

}  // namespace xc
