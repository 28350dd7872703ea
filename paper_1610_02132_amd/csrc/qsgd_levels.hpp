// Device building blocks of the quantizer by rows and columns: scales, levels, largest magnitudes.
#pragma once

#include "qsgd_layer.hpp"

namespace qsgd {

// Largest magnitude -> scale and the factor fl(127 / m); zero rows get zeros, rows with an infinity or a NaN
// the scale NaN and the factor 0.
__device__ __forceinline__ void scale_of(float m, float& scale, float& inv) {
  const bool finite = m < __builtin_huge_valf(), tiny = m < kTinyMax;
  inv = finite && !tiny ? 127.0f / m : 0.0f;
  scale = !finite ? __builtin_nanf("") : tiny ? 0.0f : m / 127.0f;
}

// Four words' bytes of one number in a word.
template <int BYTE>
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0C0C0400u | BYTE << 8 | BYTE);
  const uint32_t hi = __builtin_amdgcn_perm(d, c, 0x04000C0Cu | (uint32_t)BYTE << 24 | (uint32_t)BYTE << 16);
  return lo | hi;
}

// The levels of four values t (scaled to 127) as signed bytes of a word.  An infinity or a NaN in t (inv is 0 then, or the
// value itself) becomes level 0: the conversions to whole numbers say 0 for a NaN, and 0 times an infinity is one.
__device__ __forceinline__ uint32_t nearest_levels(const float (&t)[4]) {
  int q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = (int)__builtin_rintf(t[i]);
  return pack_bytes<0>(q[0], q[1], q[2], q[3]);
}

// floor(x) as a whole number in one instruction, 0 for a NaN.
__device__ __forceinline__ int floor_int(float x) {
  int q;
  asm("v_cvt_flr_i32_f32 %0, %1" : "=v"(q) : "v"(x));
  return q;
}

// Up iff (h + 1/2) / 65536 is below the fraction of |t|:  with F = floor(1/2 - 65536 |t|), a whole number that fp32
// holds exactly (|t| <= 127 + 2^-17, the next number after 127, so that F >= -127 * 65536 and no level passes 127),
// the level is -((F + h) >> 16).  Takes -t, whose signs say where the byte of F + h is to be negated.
__device__ __forceinline__ uint32_t stochastic_levels(const float (&minus_t)[4], const uint32_t (&h)[4]) {
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    q[i] = (uint32_t)floor_int(__builtin_fmaf(-fabsf(minus_t[i]), 65536.0f, 0.5f)) + h[i];
  const uint32_t byte = pack_bytes<2>(q[0], q[1], q[2], q[3]);
  // a byte of ones where t is positive, and the negative of those bytes: no carry leaves bit 7, which is put in last
  const uint32_t plus = __builtin_amdgcn_perm(__float_as_uint(minus_t[1]), __float_as_uint(minus_t[0]), 0x0C0C0B09u) |
                        __builtin_amdgcn_perm(__float_as_uint(minus_t[3]), __float_as_uint(minus_t[2]), 0x0B090C0Cu);
  const uint32_t flipped = byte ^ plus;
  return ((flipped & 0x7F7F7F7Fu) + (plus & 0x01010101u)) ^ (flipped & 0x80808080u);
}

// The levels of eight neighbours in a row.
template <uint32_t TYPE, bool STOCHASTIC>
__device__ __forceinline__ void eight_levels(const Eight<TYPE>& x, float inv, const HalfWords& h, uint32_t (&q)[2]) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    float t[4];
    uint32_t draw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t[i] = x.value(4 * half + i) * (STOCHASTIC ? -inv : inv);
      draw[i] = STOCHASTIC ? half_word(h, 4 * half + i) : 0;
    }
    q[half] = STOCHASTIC ? stochastic_levels(t, draw) : nearest_levels(t);
  }
}

// Magnitudes' bits, whose order is that of the magnitudes with a NaN above infinity: eight columns, two to a word for
// 16-bit types.
template <uint32_t TYPE> struct Largest {
  static constexpr int kWords = Eight<TYPE>::kWords;
  uint32_t w[kWords] = {};
  __device__ __forceinline__ void add(const Eight<TYPE>& x) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (kWords == 8) {
        w[i] = max(w[i], x.w[i] & 0x7FFFFFFFu);
      } else {
        using pair = __attribute__((ext_vector_type(2))) uint16_t;
        w[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(pair, w[i]),
                                                                      __builtin_bit_cast(pair, x.w[i] & 0x7FFF7FFFu)));
      }
    }
  }
  // ... as bits of fp32
  __device__ __forceinline__ uint32_t column(int i) const {
    Eight<TYPE> e;
#pragma unroll
    for (int j = 0; j < kWords; ++j) e.w[j] = w[j];
    return __float_as_uint(e.value(i));
  }
};

}  // namespace qsgd
