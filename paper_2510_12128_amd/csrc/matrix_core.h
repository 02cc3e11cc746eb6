// Matrix-core operands of the sequence operators (decay_attention.hip, adapter.hip): what a lane holds of a 16 x KS operand
// in LDS, for the two storage types.  gfx950 only; wave64.
//
// Lane l = 16 kg + i of a wave holds, of an operand, row (or column) i and of the KS contraction indexes those of group kg:
//   bfloat16  KS = 32, one 16x16x32 instruction, eight values a lane
//   float32   KS = 16, four 16x16x4 instructions, four values a lane, one for each
// Accumulator: column i, rows 4 kg .. 4 kg + 3.  An accumulator tile is therefore itself an operand whose contraction indexes
// are the rows of one tile (float32) or of two (bfloat16: 4 kg .. of the first tile, then 4 kg .. of the second).
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
__device__ inline uint32_t two_bf16(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
__device__ inline float from_two(uint32_t two, int nth) { return __builtin_bit_cast(float, nth ? two & 0xffff0000u : two << 16); }
// the upper halves of two float32: their first eight significant bits, the rest cut off
__device__ inline uint32_t two_upper(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
}
__device__ inline float upper(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u); }

// Two bfloat16 with zeros for those that are not finite (an exponent of ones carries into the sign's place).
__device__ inline uint32_t finite_two(uint32_t x) {
  const uint32_t odd = ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
  return x & ~(odd | (odd - (odd >> 15)));
}

// A tile in LDS whose rows are read as operands both along the rows and across them has no padding; of every row the 16-byte
// units are permuted (unit ^ swizzle(row)) so that the units that a wave's lanes want at one time lie on different banks: one unit
// of 16 consecutive rows, or some units side by side of a few rows.  Here for
// rows of that many bytes.
template <int BYTES>
__device__ inline int swizzle_bytes(int row) {
  const int far = ((row >> 3 ^ row >> 2) & 1) << 1 | (row >> 3 & 1);
  return BYTES >= 256 ? (row & 3) << 2 | far : BYTES == 128 ? (row & 2) << 1 | far : far;
}

// 16 bytes at any address that the values themselves are aligned at
__device__ inline u32x4 load16(const void* p) {
  u32x4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
// The same for loads that are waited for at once.  Those of two-byte values that are not on four bytes take a multiple of the others' time: they
// come in the five words that hold them (and no word more), shifted.
__device__ inline u32x4 load16_now(const float* p) { return load16(p); }
__device__ inline u32x4 load16_now(const uint16_t* p) {
  const uint32_t odd = (uint32_t)reinterpret_cast<uintptr_t>(p) & 2u;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(p) - odd);
  u32x4 v;
  __builtin_memcpy(&v, words, 16);
  if (odd) {
    uint32_t last;
    __builtin_memcpy(&last, words + 4, 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_alignbit(j < 3 ? v[j + 1] : last, v[j], 16);
  }
  return v;
}
// 16 bytes, or 8
template <class V>
__device__ inline void store_any(void* p, V v) {
  __builtin_memcpy(p, &v, sizeof(V));
}

struct Bf16 {
  typedef uint16_t T;
  typedef bf16x8 Frag;
  static constexpr int KS = 32;     // contraction indexes of a step
  static constexpr int E = 8;       // values in 16 bytes
  static constexpr int PARTS = 3;   // a float32 is exactly three bfloat16
  typedef u32x2 Four;               // four values
  static constexpr int SPLIT = 2;   // bfloat16 that a float32 factor beside bfloat16 ones is read as, each the nearest: 17 bits of it
  static __device__ float get(T x) { return from_bf16(x); }
  static __device__ T put(float x) { return to_bf16(x); }
  static __device__ f32x4 mfma(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

  // (Along: a 16-byte read serves lanes 0-3, 12-15, 20-23, 24-27 at one time, and three more such sets; so rows 0-3, 12-15
  // of group kg and 4-11 of the next one must differ.  Across: four rows in a row, two units or half of four units of each.
  // Measured, clocks a wave: along 4.2, against 8.0 for rows padded by 16 bytes or permuted by the row's bits exchanged.)
  template <int D>
  static __device__ int swizzle(int row) { return swizzle_bytes<2 * D>(row); }
  // Byte offsets in a tile; a lane makes its own once, and a wave's tiles and steps are constants away from it (rows that differ by
  // multiples of 16 are permuted alike).
  template <int D>
  static __device__ int unit(int row, int col) { return row * (2 * D) + (((col >> 3) ^ swizzle<D>(row)) << 4) + 2 * (col & 7); }
  // rows m0 + i, indexes k0 .. k0 + 31; `at`: unit(i, 8 kg)
  template <int D>
  static __device__ int along_at(int i, int kg) { return unit<D>(i, 8 * kg); }
  template <int D>
  static __device__ Frag along(const T* tile, int at, int m0, int k0) {
    return *reinterpret_cast<const Frag*>(reinterpret_cast<const char*>(tile) + (at ^ (2 * k0)) + m0 * 2 * D);
  }
  // rows k0 .. k0 + 31, 16 columns of which a lane's four-column run begins at `col`
  static constexpr int ACROSS = 2;
  template <int D>
  static __device__ void across_at(int (&at)[ACROSS], int col, int i, int kg) {
#pragma unroll
    for (int x = 0; x < 2; ++x) at[x] = unit<D>(8 * kg + (i >> 2) + 4 * x, col);
  }
  template <int D>
  static __device__ void columns_at(int (&at)[ACROSS], int m0, int i, int kg) { across_at<D>(at, m0 + 4 * (i & 3), i, kg); }
  template <int D>
  static __device__ Frag columns(const T* tile, const int (&at)[ACROSS], int k0, int n) {       // (16 n columns on, below 64)
    const char* p = reinterpret_cast<const char*>(tile) + k0 * 2 * D;
    return tr(p + (at[0] ^ (32 * n)), p + (at[1] ^ (32 * n)));
  }
  // the columns that accumulator tile m holds as rows (acc_row)
  template <int D>
  static __device__ void acc_columns_at(int (&at)[ACROSS], int i, int kg) { across_at<D>(at, 8 * (i & 3), i, kg); }
  template <int D>
  static __device__ Frag acc_columns(const T* tile, const int (&at)[ACROSS], int k0, int m) {
    const char* p = reinterpret_cast<const char*>(tile) + k0 * 2 * D + (m & 1) * 8;
    return tr(p + (at[0] ^ ((m >> 1) * 64)), p + (at[1] ^ ((m >> 1) * 64)));
  }
  // Index that row 4 kg of accumulator tile m stands for (4 kg + r: that plus r), so that two tiles, 2 x and 2 x + 1, are an operand
  // with contraction indexes 32 x .. in their natural order.
  static __device__ int acc_row(int m, int kg) { return (m >> 1) * 32 + 8 * kg + 4 * (m & 1); }
  static __device__ Frag row_frag(const T* row, int k0, int kg) { return *reinterpret_cast<const Frag*>(row + k0 + 8 * kg); }
  // operand whose contraction runs over the rows of a tile: columns m0 .. m0 + 15, rows k0 .. k0 + 31, by transposing reads (the
  // 16 lanes of a group read four rows of 16 columns, lane i gets column i)
  static __device__ Frag tr(const void* p0, const void* p1) {
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
  // contraction index (row of the tile) of a col_frag's value j
  static __device__ int col_k(int j, int kg) { return 8 * kg + j; }
};

struct F32 {
  typedef float T;
  typedef f32x4 Frag;
  static constexpr int KS = 16;
  static constexpr int E = 4;
  static constexpr int PARTS = 1;
  typedef f32x4 Four;
  static constexpr int SPLIT = 1;
  static __device__ float get(T x) { return x; }
  static __device__ T put(float x) { return x; }
  static __device__ f32x4 mfma(Frag a, Frag b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  // (Along: as above.  Across: four units of each of four rows, four rows apart.)
  template <int D>
  static __device__ int unit(int row, int col) {
    return row * (4 * D) + (((col >> 2) ^ (D >= 64 ? row & 15 : swizzle_bytes<4 * D>(row))) << 4) + 4 * (col & 3);
  }
  template <int D>
  static __device__ int along_at(int i, int kg) { return unit<D>(i, 4 * kg); }
  template <int D>
  static __device__ Frag along(const T* tile, int at, int m0, int k0) {
    return *reinterpret_cast<const Frag*>(reinterpret_cast<const char*>(tile) + (at ^ (4 * k0)) + m0 * 4 * D);
  }
  static constexpr int ACROSS = 4;
  template <int D>
  static __device__ void columns_at(int (&at)[ACROSS], int m0, int i, int kg) {
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = unit<D>(4 * kg + j, m0 + i);
  }
  template <int D>
  static __device__ Frag columns(const T* tile, const int (&at)[ACROSS], int k0, int n) { return acc_columns<D>(tile, at, k0, n); }
  template <int D>
  static __device__ void acc_columns_at(int (&at)[ACROSS], int i, int kg) { columns_at<D>(at, 0, i, kg); }
  template <int D>
  static __device__ Frag acc_columns(const T* tile, const int (&at)[ACROSS], int k0, int m) {
    Frag f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      f[j] = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(tile) + k0 * 4 * D + (at[j] ^ (m * 64)));
    return f;
  }
  static __device__ int acc_row(int m, int kg) { return 16 * m + 4 * kg; }
  static __device__ Frag row_frag(const T* row, int k0, int kg) { return *reinterpret_cast<const Frag*>(row + k0 + 4 * kg); }
  static __device__ Frag col_frag(const T* tile, int ld, int k0, int m0, int i, int kg) {
    const T* p = tile + (k0 + 4 * kg) * ld + m0 + i;
    return Frag{p[0], p[ld], p[2 * ld], p[3 * ld]};
  }
  static __device__ int col_k(int j, int kg) { return 4 * kg + j; }
};

// Operands of the KS / 16 accumulator tiles t[0 .. KS / 16 - 1], whose rows become the contraction index.
__device__ inline void acc_frags(const f32x4* t, F32::Frag (&out)[1], F32) { out[0] = t[0]; }
__device__ inline void acc_frags(const f32x4* t, Bf16::Frag (&out)[2], Bf16) {
  u32x4 near, rest;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float a = t[j >> 1][2 * (j & 1)], b = t[j >> 1][2 * (j & 1) + 1];
    near[j] = two_bf16(a, b);
    rest[j] = two_bf16(a - from_two(near[j], 0), b - from_two(near[j], 1));
  }
  out[0] = __builtin_bit_cast(bf16x8, near);
  out[1] = __builtin_bit_cast(bf16x8, rest);
}

// Four float32 as the operand type's numbers whose sum they are: themselves, or three bfloat16 of eight significant bits each (of an
// infinity: itself and zeros).
__device__ inline void exact_parts(f32x4 v, f32x4 (&out)[1], F32) { out[0] = v; }
__device__ inline void exact_parts(f32x4 v, u32x2 (&out)[3], Bf16) {
#pragma unroll
  for (int x = 0; x < 3; ++x) {
    out[x] = u32x2{two_upper(v[0], v[1]), two_upper(v[2], v[3])};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      v[r] -= upper(v[r]);
      v[r] = v[r] == v[r] ? v[r] : 0.f;
    }
  }
}

// The operand that the second and third parts of a factor are multiplied by: one that is not finite has its product with the first part, and the
// others may be zero.
__device__ inline F32::Frag finite_frag(F32::Frag v, F32) { return v; }
__device__ inline Bf16::Frag finite_frag(Bf16::Frag v, Bf16) {
  u32x4 x = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = finite_two(x[j]);
  return __builtin_bit_cast(bf16x8, x);
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
