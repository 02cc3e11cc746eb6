// Values of rows side by side, as a lane holds them, and the functions that the operators of state space layers apply to them.
#pragma once

#include "matrix_core.h"

namespace nugpr {

// V values of a row as they lie in memory.
template <class TR, int V>
struct Values {
  static constexpr int BYTES = V * (int)sizeof(typename TR::T), WORDS = (BYTES + 3) / 4;
  uint32_t word[WORDS];
  __device__ void clear() {
#pragma unroll
    for (int j = 0; j < WORDS; ++j) word[j] = 0;
  }
  __device__ void load_all(const typename TR::T* p) {
    if constexpr (BYTES < 4) word[0] = p[0];
    else __builtin_memcpy(word, p, BYTES);
  }
  // the first `valid` of them from p on, any number of them; the others are zero
  __device__ void load(const typename TR::T* p, int valid) {
    clear();
    if (valid >= V) {
      load_all(p);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < valid) {
          if constexpr (sizeof(typename TR::T) == 2) word[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
          else word[j] = __builtin_bit_cast(uint32_t, p[j]);
        }
    }
  }
  __device__ void store(typename TR::T* p, int valid) const {
    if (valid >= V) {
      __builtin_memcpy(p, word, BYTES);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < valid) {
          if constexpr (sizeof(typename TR::T) == 2) p[j] = (typename TR::T)(word[j >> 1] >> (16 * (j & 1)));
          else p[j] = __builtin_bit_cast(float, word[j]);
        }
    }
  }
  __device__ float get(int j) const {
    if constexpr (sizeof(typename TR::T) == 2) return from_two(word[j >> 1], j & 1);
    else return __builtin_bit_cast(float, word[j]);
  }
  __device__ void put(const float* v) {
    if constexpr (sizeof(typename TR::T) == 4) {
#pragma unroll
      for (int j = 0; j < V; ++j) word[j] = __builtin_bit_cast(uint32_t, v[j]);
    } else if constexpr (V == 1) {
      word[0] = to_bf16(v[0]);
    } else {
#pragma unroll
      for (int j = 0; j < V / 2; ++j) word[j] = two_bf16(v[2 * j], v[2 * j + 1]);
    }
  }
};

constexpr float LOG2_E = 1.44269504088896340736f, LOG2_E_REST = 1.92596299112661746887e-8f, LN_2 = 0.69314718055994530942f;

// 2^x: the instruction, good to about one rounding; zero below 2^-126
__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// e^x to about one rounding where x is float32: the exponent x log2(e) has more digits than 24 bits hold, its rest goes in as 1 + rest ln 2.
// Where x comes from a bfloat16 the product's rounding, |x| of 2^-24, is left: it is nothing beside x's own, |x| of 2^-8.
template <class TR>
__device__ inline float exp_of(float x) {
  const float y = x * LOG2_E, e = exp2_of(y);
  if constexpr (TR::E == 8) return e;
  const float rest = fmaf(x, LOG2_E_REST, fmaf(x, LOG2_E, -y));
  return fabsf(y) < 126.f ? fmaf(e * rest, LN_2, e) : e;
}

template <class TR>
__device__ inline float sigmoid_of(float x) { return __builtin_amdgcn_rcpf(1.f + exp_of<TR>(-x)); }

// log(1 + e^x) = max(x, 0) + log(1 + f), f = e^-|x| in (0, 1], and log(1 + f) = 2 artanh(s) = 2 (s + s^3 / 3 + s^5 / 5 + ..), s = f / (2 + f) <= 1/3.  The
// series from s^3 on as s q times a polynomial in q = s^2, fitted at the Chebyshev points of (0, 1/9): off by 2^-26 of the sum.  NaN stays.
template <class TR>
__device__ inline float softplus_of(float x) {
  const float f = exp_of<TR>(-fabsf(x));
  const float s = f * __builtin_amdgcn_rcpf(2.f + f), q = s * s;
  float p = fmaf(0.13433769f, q, 0.14116984f);
  p = fmaf(p, q, 0.20003835f);
  p = fmaf(p, q, 0.3333332f);
  p = fmaf(p * q, s, s);
  return fmaf(2.f, p, x > 0.f ? x : 0.f);
}

}  // namespace nugpr
