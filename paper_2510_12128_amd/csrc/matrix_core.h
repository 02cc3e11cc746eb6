// Matrix-core operands of the sequence operators (decay_attention.hip, adapter.hip): what a lane holds of a 16 x KS operand
// in LDS, for the two storage types.  gfx950 only; wave64.
//
// Lane l = 16 kg + i of a wave holds, of an operand, row (or column) i and of the KS contraction indexes those of group kg:
//   bfloat16  KS = 32, one 16x16x32 instruction, eight values a lane
//   float32   KS = 16, four 16x16x4 instructions, four values a lane, one for each
// Accumulator: column i, rows 4 kg .. 4 kg + 3.  An accumulator tile is therefore itself an operand whose contraction indexes
// are the rows of 16 (float32) or of two times 16 rows (bfloat16: 4 kg .. of the first tile, then 4 kg .. of the second).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nugpr {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// nearest bfloat16 (ties to even; NaN stays NaN)
__device__ inline uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ inline float from_bf16(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
__device__ inline uint32_t two_bf16(float lo, float hi) { return (uint32_t)to_bf16(lo) | (uint32_t)to_bf16(hi) << 16; }
// the upper halves of two float32: their first eight significant bits, the rest cut off
__device__ inline uint32_t two_upper(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
}
__device__ inline float upper(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u); }

// a 16-byte run with a value that is not finite
__device__ inline bool odd_bf16(u32x4 v) {
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) odd |= (v[j] & 0x7f80u) == 0x7f80u || (v[j] & 0x7f800000u) == 0x7f800000u;
  return odd;
}
__device__ inline bool odd_f32(u32x4 v) {
  bool odd = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) odd |= (v[j] & 0x7f800000u) == 0x7f800000u;
  return odd;
}

struct Bf16 {
  typedef uint16_t T;
  typedef bf16x8 Frag;
  static constexpr int KS = 32;     // contraction indexes of a step
  static constexpr int E = 8;       // values in 16 bytes
  static constexpr int PARTS = 3;   // a float32 is exactly three bfloat16
  static constexpr int S_PARTS = 2; // parts that a state is read with (16 of its bits)
  static __device__ float get(T x) { return from_bf16(x); }
  static __device__ T put(float x) { return to_bf16(x); }
  static __device__ bool odd(u32x4 v) { return odd_bf16(v); }
  static __device__ f32x4 mfma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

  // Rows whose contraction runs along them lie in LDS with the columns of every 32 in the order in which accumulator
  // tiles hold them: 4 kg .. 4 kg + 3 and 16 + 4 kg .. of group kg side by side.
  static __device__ int place(int col) { return (col & ~31) + ((col & 15) >> 2) * 8 + ((col >> 4) & 1) * 4 + (col & 3); }
  static __device__ void store_row(T* row, int col, u32x4 v) {        // col a multiple of 8
    T* p = row + (col & ~31) + ((col >> 3) & 1) * 16 + ((col >> 4) & 1) * 4;
    *reinterpret_cast<u32x2*>(p) = u32x2{v[0], v[1]};
    *reinterpret_cast<u32x2*>(p + 8) = u32x2{v[2], v[3]};
  }
  static __device__ Frag row_frag(const T* row, int k0, int kg) { return *reinterpret_cast<const Frag*>(row + k0 + 8 * kg); }
  // operand whose contraction runs over the rows of a tile: columns m0 .. m0 + 15, rows k0 .. k0 + 31, by transposing reads (the
  // 16 lanes of a group read four rows of 16 columns, lane i gets column i)
  static __device__ Frag tr(const T* p0, const T* p1) {
    typedef __attribute__((address_space(3))) i16x4* Lds;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p0));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p1));
    typedef short i16x8 __attribute__((ext_vector_type(8)));
    const i16x8 r = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(Frag, r);
  }
  static __device__ Frag col_frag(const T* tile, int ld, int k0, int m0, int i, int kg) {
    const T* p = tile + (k0 + 8 * kg + (i >> 2)) * ld + m0 + 4 * (i & 3);
    return tr(p, p + 4 * ld);
  }
  // the same of rows stored by store_row
  static __device__ Frag col_frag_placed(const T* tile, int ld, int k0, int m0, int i, int kg) {
    const T* p = tile + (k0 + 8 * kg + (i >> 2)) * ld + (m0 & ~31) + (i & 3) * 8 + ((m0 >> 4) & 1) * 4;
    return tr(p, p + 4 * ld);
  }
  // contraction index (row of the tile) of a col_frag's value j
  static __device__ int col_k(int j, int kg) { return 8 * kg + j; }
};

struct F32 {
  typedef float T;
  typedef f32x4 Frag;
  static constexpr int KS = 16;
  static constexpr int E = 4;
  static constexpr int PARTS = 1;
  static constexpr int S_PARTS = 1;
  static __device__ float get(T x) { return x; }
  static __device__ T put(float x) { return x; }
  static __device__ bool odd(u32x4 v) { return odd_f32(v); }
  static __device__ f32x4 mfma(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  static __device__ int place(int col) { return col; }
  static __device__ void store_row(T* row, int col, u32x4 v) { *reinterpret_cast<u32x4*>(row + col) = v; }
  static __device__ Frag row_frag(const T* row, int k0, int kg) { return *reinterpret_cast<const Frag*>(row + k0 + 4 * kg); }
  static __device__ Frag col_frag(const T* tile, int ld, int k0, int m0, int i, int kg) {
    const T* p = tile + (k0 + 4 * kg) * ld + m0 + i;
    return Frag{p[0], p[ld], p[2 * ld], p[3 * ld]};
  }
  static __device__ Frag col_frag_placed(const T* tile, int ld, int k0, int m0, int i, int kg) {
    return col_frag(tile, ld, k0, m0, i, kg);
  }
  static __device__ int col_k(int j, int kg) { return 4 * kg + j; }
};

// Operand(s) of accumulator tiles: the KS / 16 tiles t[0 .. KS / 16 - 1], whose rows become the contraction index.
__device__ inline void acc_frags(const f32x4* t, F32::Frag (&out)[1], F32) { out[0] = t[0]; }
__device__ inline void acc_frags(const f32x4* t, Bf16::Frag (&out)[2], Bf16) {
  u32x4 hi, lo;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = t[j >> 1][2 * (j & 1)], b = t[j >> 1][2 * (j & 1) + 1];
    hi[j] = two_upper(a, b);
    lo[j] = two_bf16(a - upper(a), b - upper(b));
  }
  out[0] = __builtin_bit_cast(bf16x8, hi);
  out[1] = __builtin_bit_cast(bf16x8, lo);
}

// Operand times one float32 weight a contraction index, without rounding to fewer than 24 bits: in bfloat16 the product is cut
// into three numbers of eight significant bits each.
__device__ inline void weighted_frags(F32::Frag v, const float* w, F32::Frag (&out)[1], F32) {
#pragma unroll
  for (int j = 0; j < 4; ++j) out[0][j] = v[j] * w[j];
}
__device__ inline void weighted_frags(Bf16::Frag v, const float* w, Bf16::Frag (&out)[3], Bf16) {
  const u32x4 raw = __builtin_bit_cast(u32x4, v);
  u32x4 p[3];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float a = __builtin_bit_cast(float, raw[j] << 16) * w[2 * j];
    float b = __builtin_bit_cast(float, raw[j] & 0xffff0000u) * w[2 * j + 1];
    p[0][j] = two_upper(a, b);
    a -= upper(a);
    b -= upper(b);
    p[1][j] = two_upper(a, b);
    p[2][j] = two_upper(a - upper(a), b - upper(b));
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) out[k] = __builtin_bit_cast(bf16x8, p[k]);
}

}  // namespace nugpr
