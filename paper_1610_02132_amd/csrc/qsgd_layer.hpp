// Argument blocks, launchers and device building blocks of the operators of a layer in 8 bits
// (internal to libqsgd).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "qsgd.h"
#include "qsgd_device.hpp"

namespace qsgd {

// Key and position of a matrix's draws (see qsgd_draws).
struct DrawArgs {
  uint32_t key0, key1, stream_id, iteration, row_base;
  const uint32_t* iteration_dev;
};

// The eight half-words of the block that holds the draws of columns 8 * c8 .. 8 * c8 + 7 of a row.
struct HalfWords { uint32_t w[4]; };
__device__ __forceinline__ uint32_t half_word(const HalfWords& h, int i) {
  return i & 1 ? h.w[i >> 1] >> 16 : h.w[i >> 1] & 0xFFFFu;
}
__device__ __forceinline__ uint32_t draw_iteration(const DrawArgs& d) {
  return d.iteration + (d.iteration_dev ? *d.iteration_dev : 0u);
}
__device__ __forceinline__ HalfWords draw_block(const DrawArgs& d, uint32_t iteration, uint32_t row, uint32_t c8) {
  HalfWords h;
  philox4x32_10(c8, d.row_base + row, d.stream_id, iteration, d.key0, d.key1, h.w);
  return h;
}

// Several blocks at once: the key is stepped once for all of them, and products of words that they share are made once.
template <int N>
__device__ __forceinline__ void draw_blocks(const DrawArgs& d, uint32_t iteration, const uint32_t (&row)[N],
                                            const uint32_t (&c8)[N], HalfWords* h) {
  uint32_t c1[N], out[N][4];
#pragma unroll
  for (int i = 0; i < N; ++i) c1[i] = d.row_base + row[i];
  philox4x32_10_xn<N>(c8, c1, d.stream_id, iteration, d.key0, d.key1, out);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) h[i].w[j] = out[i][j];
}

// ---- element types ---------------------------------------------------------------
// A value's bits, their fp32 value, and fp32 rounded to the type (nearest, ties to even).
template <uint32_t TYPE> struct Element;
template <> struct Element<QSGD_TYPE_F32> {
  using bits = uint32_t;
  __device__ static float widen(uint32_t b) { return __uint_as_float(b); }
  __device__ static uint32_t narrow(float v) { return __float_as_uint(v); }
};
template <> struct Element<QSGD_TYPE_BF16> {
  using bits = uint16_t;
  __device__ static float widen(uint32_t b) { return __uint_as_float(b << 16); }
  __device__ static uint32_t narrow(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  __device__ static uint32_t narrow2(float v, float w) {   // two values in a word
    using values = __attribute__((ext_vector_type(2))) float;
    using pair = __attribute__((ext_vector_type(2))) __bf16;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((values{v, w}), pair));
  }
};
template <> struct Element<QSGD_TYPE_F16> {
  using bits = uint16_t;
  __device__ static float widen(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }
  __device__ static uint32_t narrow(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
  __device__ static uint32_t narrow2(float v, float w) { return narrow(v) | narrow(w) << 16; }
};

// Eight neighbouring elements: 16 bytes of a 16-bit type, 32 of fp32.
template <uint32_t TYPE> struct Eight {
  static constexpr int kWords = 2 * (int)sizeof(typename Element<TYPE>::bits);
  uint32_t w[kWords];
  __device__ __forceinline__ uint32_t bits(int i) const {
    if constexpr (kWords == 8) return w[i];
    else return i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
  }
  __device__ __forceinline__ float value(int i) const { return Element<TYPE>::widen(bits(i)); }
  __device__ __forceinline__ void set(int i, uint32_t b) {
    if constexpr (kWords == 8) w[i] = b;
    else w[i >> 1] = i & 1 ? w[i >> 1] | b << 16 : b;   // (in ascending order)
  }
  // Elements [0, n) of p, aligned to their own size (the machine loads 16 bytes from any address); the others read as
  // zero.  STREAM: past the caches, for matrices that they do not hold.
  using Words = __attribute__((ext_vector_type(4), aligned(sizeof(typename Element<TYPE>::bits)))) uint32_t;
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const void* p, uint32_t n) {
    if (n >= 8) {
#pragma unroll
      for (int j = 0; j < kWords; j += 4) {
        const Words* from = reinterpret_cast<const Words*>(p) + j / 4;
        const Words v = STREAM ? __builtin_nontemporal_load(from) : *from;
        w[j] = v.x; w[j + 1] = v.y; w[j + 2] = v.z; w[j + 3] = v.w;
      }
    } else {
      const auto* e = reinterpret_cast<const typename Element<TYPE>::bits*>(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) set(i, (uint32_t)i < n ? e[i] : 0u);
    }
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void store(void* p, uint32_t n) const {
    if (n >= 8) {
#pragma unroll
      for (int j = 0; j < kWords; j += 4) {
        Words* to = reinterpret_cast<Words*>(p) + j / 4;
        const Words v = {w[j], w[j + 1], w[j + 2], w[j + 3]};
        if constexpr (STREAM) __builtin_nontemporal_store(v, to);
        else *to = v;
      }
    } else {
      auto* e = reinterpret_cast<typename Element<TYPE>::bits*>(p);
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if ((uint32_t)i < n) e[i] = (typename Element<TYPE>::bits)bits(i);
    }
  }
};

template <uint32_t TYPE>
__device__ __forceinline__ const void* element_at(const void* base, uint64_t ld, uint32_t r, uint32_t c) {
  return reinterpret_cast<const typename Element<TYPE>::bits*>(base) + (r * ld + c);
}
template <uint32_t TYPE>
__device__ __forceinline__ void* element_at(void* base, uint64_t ld, uint32_t r, uint32_t c) {
  return reinterpret_cast<typename Element<TYPE>::bits*>(base) + (r * ld + c);
}

// ---- dropout -----------------------------------------------------------------------
struct DropoutArgs {
  const void *x, *residual;   // residual: or null
  void* y;
  uint64_t x_ld, residual_ld, y_ld;
  uint32_t rows, cols;
  uint32_t drop;              // D: draws below it drop the element
  float scale;                // 65536 / (65536 - D), or 0
  DrawArgs draws;
};
hipError_t launch_dropout(const DropoutArgs& a, uint32_t type, hipStream_t st);

// ---- quantizer ---------------------------------------------------------------------
constexpr float kTinyMax = 0x1p-119f;   // rows whose largest magnitude is below it count as zero: 127 / m and m / 127 stay normal

struct QuantizeArgs {
  const void* x;
  uint64_t ld;
  uint32_t rows, cols;
  DrawArgs draws;
  int8_t* q_rows; uint64_t q_rows_ld; float* row_scale;   // row_scale: or null
  int8_t* q_cols; uint64_t q_cols_ld; float* col_scale;
  // workspace of the column form
  uint32_t strip_lanes, chunks, chunk_rows;
  uint32_t* part_max;         // chunks x cols: largest magnitude's bits as fp32; or null: no column form
  float* part_sum;            // chunks x cols, or null: sums of the columns
  float* col_sum;             // where the sums go
  // workgroups (plan_quantize)
  uint32_t row_lanes, row_blocks, max_blocks, tile_blocks;
  bool stream;                // the second launch reads x past the caches
  bool shared_lines;          // rows do not start at lines of 128 bytes
  uint32_t tile_rows;         // rows that a workgroup of the second launch takes, a multiple of 128
};
struct QuantizeJobs { uint32_t count, blocks[2]; QuantizeArgs job[3]; };   // blocks: of the two launches
// Lanes to a row of a strip of columns, rows of a chunk, and how many chunks there are.
void plan_columns(uint32_t rows, uint32_t cols, uint32_t& strip_lanes, uint32_t& chunks, uint32_t& chunk_rows);
// As many numbers, chunks times columns, as these sizes or any smaller ones have at most.
uint64_t column_numbers(uint64_t rows, uint64_t cols);
// Fills in the workgroups of both launches and says how many the larger one has.
uint64_t plan_quantize(QuantizeJobs& jobs, uint32_t type);
// First launch: row forms, and the columns' maxima and sums; second: column forms.
hipError_t launch_quantize(const QuantizeJobs& jobs, uint32_t type, bool stochastic, hipStream_t st, bool second);

// ---- product -----------------------------------------------------------------------
struct ProductArgs {
  const int8_t *a, *b;
  uint64_t a_ld, b_ld;        // multiples of 16, below 2^23
  uint32_t M, N, K;
  const float *a_scale, *b_scale, *bias;   // bias: or null
  void* y;
  uint64_t y_ld;
  uint32_t type;
  uint32_t splits, split_k;   // pieces of K and their length (a multiple of the tile's depth)
  int32_t* part;              // splits x M x N sums, or null with one piece
};
enum ProductKind : uint32_t {
  kProductFew,        // at most 32 rows of a
  kProductTile64Deep, // tiles of 64 x 64 results, four stages of k, ...
  kProductTile64,     // ... and two
  kProductTile128,
  kProductTile128x64,
  kProductTile256,
  kProductShallow,    // little depth, straight from memory, one piece
};
struct ProductPlan { uint32_t kind, splits, split_k; uint64_t bytes; };
// One product, or two that are planned alike and in one piece each.
struct ProductPair { ProductArgs of[2]; uint32_t count, first; };
ProductPlan plan_product(uint32_t M, uint32_t N, uint32_t K);
// Bytes of workspace that are enough for a product of these sizes and for any of smaller ones.
uint64_t product_space(uint64_t M, uint64_t N, uint64_t K);
hipError_t launch_products(const ProductPair& pair, uint32_t kind, hipStream_t st);
// The layer on few tokens, x quantized on the way: product has no a and no a_scale.
struct LinearArgs {
  ProductArgs product;
  const void* x;
  uint64_t x_ld;
  DrawArgs draws;
};
bool linear_few_fits(uint32_t M, uint32_t N, uint32_t K);
hipError_t launch_linear_few(const LinearArgs& l, uint32_t type, bool stochastic, hipStream_t st);
hipError_t launch_product_join(const ProductArgs& a, hipStream_t st);

}  // namespace qsgd
