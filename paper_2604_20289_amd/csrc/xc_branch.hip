// Attention of branching sequences over paged keys and values:
// o = softmax(scale q k^T) v over all keys of the row's sequence.
//
// The work is cut on the host (plan_attention): a unit is up to 256 query rows
// (float32: 128) over a run of keys of one page table.  The rows of a unit are
// (batch row, query head of one key head); for a shared history they come
// from many sequences, which is how its keys are read once for all of them.
// A row whose keys lie in several units gets its pieces merged.
//
// bf16 kernel: 8 waves of 32 query rows.  As in the model's own attention,
// S^T = K Q^T on v_mfma_f32_32x32x16_bf16 puts one query's scores into one
// lane, and the K rows sit permuted in LDS so that a lane's scores are the 8
// consecutive keys its operand of O^T += V^T P^T wants.  What differs:
//   * pages hold V row-major (one token is one contiguous write, a page copy
//     is one run), so its operand is formed by the transposing LDS read;
//   * tiles of 64 places come through the page table: a 16-place group lies in
//     one page, so the DMA of 8 rows has a wave-uniform 64-bit base.  A wave
//     keeps 64 table entries in a register and reads them by lane;
//   * places outside the unit's keys are not read: their lanes fetch the
//     nearest valid place, and the scores are masked.
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

constexpr int kXcds = 8;  // each has its own L2
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

// (unit, key head) of a workgroup: heads outermost, dealt to the XCDs in
// contiguous ranges, so that the workgroups of one XCD read the same keys
__device__ __forceinline__ bool unit_of(const AttnArgs& a, int& u, int& h) {
  const int total = a.n_units * a.buf.kv_heads;
  const int per_xcd = (total + kXcds - 1) / kXcds;
  const int i = (blockIdx.x % kXcds) * per_xcd + blockIdx.x / kXcds;
  if ((int)(blockIdx.x / kXcds) >= per_xcd || i >= total) return false;
  h = i / a.n_units;
  u = i - h * a.n_units;
  return true;
}

// Where a query row's results go.
struct RowOut {
  long long out, piece, stat;
};
__device__ __forceinline__ RowOut row_out(const AttnArgs& a, const AttnUnit& un, int h, int r) {
  const int t = un.tok0 + r / a.group, qh = h * a.group + r % a.group;
  RowOut o;
  o.out = (long long)t * a.out_ld + qh * a.buf.D;
  o.stat = ((long long)un.slot * a.rows + t) * a.q_heads + qh;
  o.piece = o.stat * a.buf.D;
  return o;
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, 1) void branch_attn_bf16_kernel(AttnArgs a) {
  constexpr int KCG = D / 64;             // 1 KB blocks per 8 rows
  constexpr int NB = 8 * KCG / kWaves;    // blocks per wave, of a K or a V tile
  constexpr int DT = D / 32, KS = D / 16;
  // LDS tiles in 1 KB blocks of 8 rows x 8 sixteen-byte chunks.  K: row r,
  // chunk c at ((c % 8) ^ (r / 8 % 2)) * 8 + r % 8: the 16 rows that a quarter
  // wave reads at one chunk fall into 16 bank groups.  V: (r / 4 % 2 * 8 + c) *
  // 4 + r % 4: the 4 rows x 4 chunks that half a wave of a transposing read
  // takes are 256 contiguous bytes.
  __shared__ __attribute__((aligned(1024))) char sK0[64 * D * 2];
  __shared__ __attribute__((aligned(1024))) char sK1[64 * D * 2];
  __shared__ __attribute__((aligned(1024))) char sK2[64 * D * 2];
  __shared__ __attribute__((aligned(1024))) char sV0[64 * D * 2];
  __shared__ __attribute__((aligned(1024))) char sV1[64 * D * 2];
  __shared__ __attribute__((aligned(1024))) char sV2[64 * D * 2];
  int u, h;
  if (!unit_of(a, u, h)) return;
  const AttnUnit un = a.units[u];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const int rows = un.tokens * a.group;
  const int base = un.lo & ~15, n = (un.hi - base + 63) >> 6, last = un.hi - 1;
  const bool live = wave * 32 < rows;
  const int shift = a.buf.shift, in_page = (1 << shift) - 1;
  const long long head_bytes = (long long)D * 2 << shift, page_bytes = head_bytes * a.buf.kv_heads;
  const char* Kh = reinterpret_cast<const char*>(a.buf.keys) + h * head_bytes;
  const char* Vh = reinterpret_cast<const char*>(a.buf.values) + h * head_bytes;

  // the unit's page table, 64 entries at a time: entry e0 + lane
  const int* table = a.tables + un.table;
  const int e_last = last >> shift;
  int e0 = un.lo >> shift;
  int entries = table[min(e0 + lane, e_last)];

  // block i of this wave: rows 8 rg .. of the tile, all in the 16-place group rg / 2
  int k_row[NB], v_row[NB];
  unsigned k_col[NB], v_col[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int B = wave + kWaves * i, rg = B / KCG, cg = B % KCG;
    const int R = rg * 8 + (lane & 7);
    k_row[i] = key_of_row(R >> 5, R & 31);
    k_col[i] = (cg * 8 + ((lane >> 3) ^ (rg & 1))) * 16;
    v_row[i] = rg * 8 + (lane >> 5) * 4 + (lane & 3);
    v_col[i] = (cg * 8 + ((lane >> 2) & 7)) * 16;
  }
  auto fetch = [&](const char* buf, int j, int row, unsigned col, char* dst) __attribute__((always_inline)) {
    const int at = min(max(base + j * 64 + row, un.lo), last);
    const int e = __builtin_amdgcn_readfirstlane(at >> shift) - e0;
    const long long page = __builtin_amdgcn_readlane(entries, e);
    dma16(buf + page * page_bytes, (unsigned)(at & in_page) * (D * 2) + col, dst);
  };
  auto dma_k = [&](int j, char* dst) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) fetch(Kh, j, k_row[i], k_col[i], dst + (wave + kWaves * i) * 1024);
  };
  auto dma_v = [&](int j, char* dst) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) fetch(Vh, j, v_row[i], v_col[i], dst + (wave + kWaves * i) * 1024);
  };
  // the register's entries cover tile j (the next V) to tile j + 1 (the next K)
  auto cover = [&](int j) __attribute__((always_inline)) {
    const int top = min(base + j * 64 + 127, last) >> shift;
    if (top - e0 >= 64) {
      e0 = max(base + j * 64, un.lo) >> shift;
      entries = table[min(e0 + lane, e_last)];
      asm volatile("" : "+v"(entries));  // waited for here, not in the loop
    }
  };

  dma_k(0, sK0);
  dma_v(0, sV0);
  if (n > 1) dma_k(1, sK1), dma_v(1, sV1);
  if (n > 2) dma_k(2, sK2);

  bf16x8 qf[KS];
  if (live) {
    const int r = min(wave * 32 + lo, rows - 1);
    const bf16* q = reinterpret_cast<const bf16*>(a.q) + (un.tok0 + r / a.group) * a.q_ld +
                    (long long)(h * a.group + r % a.group) * D + hi * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(q + ks * 16);
  }
  f32x16 oacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  const int k_frag = (lo >> 3) * KCG * 1024 + (hi ^ ((lo >> 3) & 1)) * 128 + (lo & 7) * 16;
  const int v_frag = hi * KCG * 1024 + (((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) * 64 + ((lane >> 2) & 3) * 16 +
                     (lane & 1) * 8;
  auto qk = [&](f32x16 (&s)[2], const char* kt) __attribute__((always_inline)) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        const bf16x8 k = *reinterpret_cast<const bf16x8*>(kt + k_frag + mt * 4 * KCG * 1024 + (ks >> 2) * 1024 +
                                                          (ks & 3) * 256);
        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[ks], s[mt], 0, 0, 0);
      }
  };
  auto v_half = [&](const char* vt, int off) __attribute__((always_inline)) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + v_frag + off));
  };
  auto pv = [&](const bf16x8 (&p)[4], const char* vt) __attribute__((always_inline)) {
#pragma unroll
    for (int kv = 0; kv < 4; ++kv)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int off = kv * 2 * KCG * 1024 + (dt >> 1) * 1024 + (dt & 1) * 256;
        const s16x8 v = __builtin_shufflevector(v_half(vt, off), v_half(vt, off + 512), 0, 1, 2, 3, 4, 5, 6, 7);
        oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p[kv], oacc[dt], 0, 0, 0);
      }
  };
  auto mask = [&](f32x16 (&s)[2], int j) __attribute__((always_inline)) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = base + j * 64 + key_of_row(mt, (i >> 2) * 8 + hi * 4 + (i & 3));
        if (at < un.lo || at > last) s[mt][i] = -INFINITY;
      }
  };
  // The running maximum moves only when a tile's maximum exceeds it by more
  // than 8: p stays <= 2^8 in between, which float sums and bf16 carry.
  auto update_max = [&](const f32x16 (&s)[2]) __attribute__((always_inline)) {
    float mx = s[0][0];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[mt][i]);
    mx = partner_max(mx) * a.scale;
    if (mx > m_run + 8.0f) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
      m_run = mx;
    }
  };
  // p = 2^(scale s - m), rounded to bf16 for the matrix cores (2^-9 each, of
  // either sign); the sum takes them before that rounding
  auto probs = [&](f32x16 (&s)[2], bf16x8 (&p)[4]) __attribute__((always_inline)) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][i], a.scale, -m_run));
        sum[i & 3] += e;
        p[mt * 2 + (i >> 3)][i & 7] = (bf16)e;
      }
    l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };

  // tile 0 has landed once at most K(1), V(1), K(2) are in flight (V(0) is
  // waited for with K(1) below)
  XC_WAIT_VM(0);
  tile_barrier();
  f32x16 sa[2], sb[2];
  if (live) {
    qk(sa, sK0);
    mask(sa, 0);
    update_max(sa);
  }
  tile_barrier();  // S(0) has read K(0): its slot may be refilled

  // Tile j: S(j + 1) on the matrix cores beside the softmax of S(j), then
  // O += P(j) V(j).  K(j + 3) and V(j + 2) are requested into the slots that
  // tile j - 1 was the last to read; what was requested one tile earlier has
  // landed when the tile ends.
  auto iter = [&](int j, f32x16 (&s)[2], f32x16 (&sn)[2], const char* kn, const char* vt, char* kd, char* vd)
      __attribute__((always_inline)) {
    if (j + 2 < n) cover(j + 2);
    if (j + 3 < n) dma_k(j + 3, kd);
    if (j + 2 < n) dma_v(j + 2, vd);
    if (live) {
      if (j + 1 < n) qk(sn, kn);
      bf16x8 p[4];
      probs(s, p);
      pv(p, vt);
      if (j + 1 < n) {
        if (j + 2 == n) mask(sn, j + 1);
        update_max(sn);
      }
    }
    if (j + 3 < n) { XC_WAIT_VM(2 * NB); } else { XC_WAIT_VM(0); }
    tile_barrier();
  };
  for (int j = 0; j < n; j += 6) {
    iter(j, sa, sb, sK1, sV0, sK0, sV2);
    if (j + 1 < n) iter(j + 1, sb, sa, sK2, sV1, sK1, sV0);
    if (j + 2 < n) iter(j + 2, sa, sb, sK0, sV2, sK2, sV1);
    if (j + 3 < n) iter(j + 3, sb, sa, sK1, sV0, sK0, sV2);
    if (j + 4 < n) iter(j + 4, sa, sb, sK2, sV1, sK1, sV0);
    if (j + 5 < n) iter(j + 5, sb, sa, sK0, sV2, sK2, sV1);
  }
  if (!live) return;
  const int r = wave * 32 + lo;
  const float l = partner_sum(l_run);
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

// float32: the same division of the work with 4 waves of 32 query rows and
// tiles of 32 keys on v_mfma_f32_32x32x2_f32.  The two k indices of a product
// are any two head dims (S) or keys (P V) as long as both operands agree, so
// the operands need no shuffles: S takes dims 8 t + e and 8 t + 4 + e, P V the
// two keys whose scores sit in one register of the two half-waves.
constexpr int kWavesF32 = 4;
template <int D>
__global__ __launch_bounds__(64 * kWavesF32, 1) void branch_attn_f32_kernel(AttnArgs a) {
  constexpr int LD = D + 4;  // 16-byte reads down a column then meet different banks
  constexpr int DT = D / 32, CH = D / 4, PER = 32 * CH / (64 * kWavesF32);
  __shared__ __attribute__((aligned(16))) float sK[2][32 * LD], sV[2][32 * LD];
  int u, h;
  if (!unit_of(a, u, h)) return;
  const AttnUnit un = a.units[u];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hi = lane >> 5, lo = lane & 31;
  const int rows = un.tokens * a.group;
  const int n = (un.hi - un.lo + 31) >> 5, last = un.hi - 1;
  const bool live = wave * 32 < rows;
  const int shift = a.buf.shift;
  const float* K = reinterpret_cast<const float*>(a.buf.keys);
  const float* V = reinterpret_cast<const float*>(a.buf.values);
  const int* table = a.tables + un.table;

  f32x4 kr[PER], vr[PER];
  auto load = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = tid + 64 * kWavesF32 * i;
      const int at = min(un.lo + j * 32 + c / CH, last);
      const long long page = table[at >> shift];
      const long long o = (((page * a.buf.kv_heads + h) << shift) + (at & ((1 << shift) - 1))) * D + c % CH * 4;
      kr[i] = *reinterpret_cast<const f32x4*>(K + o);
      vr[i] = *reinterpret_cast<const f32x4*>(V + o);
    }
  };
  auto store = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = tid + 64 * kWavesF32 * i;
      *reinterpret_cast<f32x4*>(&sK[b][c / CH * LD + c % CH * 4]) = kr[i];
      *reinterpret_cast<f32x4*>(&sV[b][c / CH * LD + c % CH * 4]) = vr[i];
    }
  };
  load(0);
  f32x4 qf[D / 8];
  if (live) {
    const int r = min(wave * 32 + lo, rows - 1);
    const float* q = reinterpret_cast<const float*>(a.q) + (un.tok0 + r / a.group) * a.q_ld +
                     (long long)(h * a.group + r % a.group) * D + hi * 4;
#pragma unroll
    for (int t = 0; t < D / 8; ++t) qf[t] = *reinterpret_cast<const f32x4*>(q + t * 8);
  }
  f32x16 oacc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  store(0);
  __syncthreads();
  for (int j = 0; j < n; ++j) {
    const int b = j & 1;
    if (j + 1 < n) load(j + 1);
    if (live) {
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
      for (int t = 0; t < D / 8; ++t) {
        const f32x4 k = *reinterpret_cast<const f32x4*>(&sK[b][lo * LD + t * 8 + hi * 4]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], qf[t][e], s, 0, 0, 0);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        // only the unit's last tile reaches past its keys
        if (un.lo + j * 32 + (i >> 2) * 8 + hi * 4 + (i & 3) > last) s[i] = -INFINITY;
        mx = fmaxf(mx, s[i]);
      }
      mx = partner_max(mx) * a.scale;
      if (mx > m_run) {
        const float alpha = exp2f(m_run - mx);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
        m_run = mx;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = exp2f(__builtin_fmaf(s[i], a.scale, -m_run));
        l_run += s[i];
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(
              sV[b][((i >> 2) * 8 + hi * 4 + (i & 3)) * LD + dt * 32 + lo], s[i], oacc[dt], 0, 0, 0);
    }
    if (j + 1 < n) store(b ^ 1);
    __syncthreads();
  }
  if (!live) return;
  const int r = wave * 32 + lo;
  const float l = partner_sum(l_run);
  if (r >= rows) return;
  const RowOut o = row_out(a, un, h, r);
  const float inv = un.slot < 0 ? 1.0f / l : 1.0f;
  float* row = un.slot < 0 ? reinterpret_cast<float*>(a.out) + o.out : a.pieces + o.piece;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = oacc[dt][g * 4 + i] * inv;
      *reinterpret_cast<f32x4*>(row + dt * 32 + g * 8 + hi * 4) = v;
    }
  if (un.slot >= 0 && hi == 0) a.stats[o.stat] = make_float2(m_run, l);
}

// Joins the pieces of each (row, query head), in slot order:
// O = sum_p w_p O_p / sum_p w_p l_p, w_p = 2^(m_p - max m).
// D / 4 lanes own one of them, four head dims each.
template <typename T, int D>
__global__ __launch_bounds__(256) void branch_merge_kernel(AttnArgs a) {
  constexpr int LPH = D / 4;
  const long long i = (long long)blockIdx.x * (256 / LPH) + threadIdx.x / LPH;
  const int d0 = threadIdx.x % LPH * 4;
  const long long rq = (long long)a.rows * a.q_heads;
  if (i >= rq) return;
  const int t = (int)(i / a.q_heads);
  const OwnSlots own = a.own[t];
  const int n = a.shared_slots + own.n;
  if (n == 0) return;  // written by its only unit
  auto slot = [&](int p) __attribute__((always_inline)) {
    return (long long)(p < a.shared_slots ? p : own.first + p - a.shared_slots) * rq + i;
  };
  float m = -INFINITY;
  for (int p = 0; p < n; ++p) m = fmaxf(m, a.stats[slot(p)].x);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f;
  for (int p = 0; p < n; ++p) {
    const long long at = slot(p);
    const float2 st = a.stats[at];
    const f32x4 o = *reinterpret_cast<const f32x4*>(a.pieces + at * D + d0);
    const float w = exp2f(st.x - m);
    den += w * st.y;
    acc += w * o;
  }
  T* out = reinterpret_cast<T*>(a.out) + t * a.out_ld + (i - (long long)t * a.q_heads) * D + d0;
  const float inv = 1.0f / den;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (T)(acc[e] * inv);
}

}  // namespace

// Requirements (the caller's): D in {64, 128} (float32: 32 too); every unit
// has at least one key and at most attn_tile_rows query rows; page tables,
// slots and piece buffers cover what the units name.
hipError_t launch_branch_attention(int dtype, const AttnArgs& a, hipStream_t st) {
  const int total = a.n_units * a.buf.kv_heads, D = a.buf.D;
  if (total == 0) return hipSuccess;
  const int grid = (total + kXcds - 1) / kXcds * kXcds;
  if (dtype == 1) {
    if (D == 128) branch_attn_bf16_kernel<128><<<grid, 64 * kWaves, 0, st>>>(a);
    else branch_attn_bf16_kernel<64><<<grid, 64 * kWaves, 0, st>>>(a);
  } else {
    if (D == 128) branch_attn_f32_kernel<128><<<grid, 64 * kWavesF32, 0, st>>>(a);
    else if (D == 64) branch_attn_f32_kernel<64><<<grid, 64 * kWavesF32, 0, st>>>(a);
    else branch_attn_f32_kernel<32><<<grid, 64 * kWavesF32, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_slots == 0) return e;
  const long long per = 256 / (D / 4), rq = (long long)a.rows * a.q_heads;
  const unsigned mg = (unsigned)((rq + per - 1) / per);
#define XC_MERGE(T, DD) branch_merge_kernel<T, DD><<<mg, 256, 0, st>>>(a)
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
