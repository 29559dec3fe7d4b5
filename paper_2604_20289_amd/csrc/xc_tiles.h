// Tiles of the branching cache's matrix kernels: how keys, values and queries
// lie in LDS, how they come there, and what of a tile a row sees.  Device code.
#pragma once

#include <hip/hip_runtime.h>

namespace xc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// MFMA row R of a 32-key half tile -> key offset within the 64-key tile, as the attention has its keys
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

// What a query row sees of a run of places: [begin, end) and [lo, sink_end).
struct Limits {
  int begin, end, lo, sink_end;
  __device__ __forceinline__ bool sees(int at) const { return (at >= begin && at < end) || (at >= lo && at < sink_end); }
  // of 32 places from `at` on, a bit each
  __device__ __forceinline__ unsigned bits(int at) const {
    auto below = [](int n) __attribute__((always_inline)) { return n <= 0 ? 0u : ~0u >> (32 - min(n, 32)); };
    return (below(end - at) & ~below(begin - at)) | (below(sink_end - at) & ~below(lo - at));
  }
};
// Scores of a half tile at `at` that the row does not see: -infinity.  Bits
// and not comparisons: these would want a pair of scalar registers each.
// key(i): where the i-th of a lane's 16 scores lies, `bits` moved to its half wave's.
template <typename Key>
__device__ __forceinline__ void mask_row(f32x16& s, unsigned bits, Key key) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const unsigned keep = (unsigned)((int)(bits << (31 - key(i))) >> 31);
    s[i] = __uint_as_float((__float_as_uint(s[i]) & keep) | (0xff800000u & ~keep));
  }
}
__device__ __forceinline__ void mask_row(f32x16& s, int at, int hi, const Limits& lim) {
  mask_row(s, lim.bits(at) >> (hi * 8), [](int i) { return key_of_row(0, (i >> 2) * 8 + (i & 3)); });
}

}  // namespace xc
