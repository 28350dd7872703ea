// Quantizer Q_s of Sec. 3.1 (Eq. 2) with s = 127 and max scaling (Sec. 4), a bucket being a row or a
// column of a matrix, levels as signed bytes.  Memory bound: the row form reads a row once more than
// it has to (from the cache), the column form reads the matrix twice (maxima, then levels, which leave
// transposed through LDS).
#include "qsgd_layer.hpp"

namespace qsgd {
namespace {

// Largest magnitude -> scale and the factor fl(127 / m); zero rows get zeros, rows with an infinity or a NaN
// the scale NaN and levels 0.
__device__ __forceinline__ void scale_of(float m, float& scale, float& inv) {
  const bool finite = m < __builtin_huge_valf(), tiny = m < kTinyMax;
  inv = finite && !tiny ? 127.0f / m : 0.0f;
  scale = !finite ? __builtin_nanf("") : tiny ? 0.0f : m / 127.0f;
}

// The level of one value as a signed byte.
__device__ __forceinline__ uint32_t level_of(float v, float inv, bool stochastic, uint32_t h) {
  // a row that holds an infinity or a NaN has inv = 0 and products that are NaN, else |t| <= 127 (1 + 2^-23)
  const float t = inv > 0.0f ? v * inv : 0.0f;
  int level;
  if (stochastic) {
    const float a = fabsf(t), low = floorf(a), u = ((float)h + 0.5f) * 0x1p-16f;
    level = min((int)low + (u < a - low ? 1 : 0), 127);
    level = t < 0.0f ? -level : level;
  } else {
    level = (int)rintf(t);
  }
  return (uint32_t)level & 0xFFu;
}

// The larger of two magnitudes by their bits: a NaN's are above infinity's.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_quantize_rows(QuantizeArgs a) {
  const uint32_t r = blockIdx.x, c8s = (a.cols + 7) / 8, iteration = draw_iteration(a.draws);
  __shared__ uint32_t part[4];
  uint32_t m = 0;
  for (uint32_t c8 = threadIdx.x; c8 < c8s; c8 += 256) {
    Eight<TYPE> x;
    x.load(element_at<TYPE>(a.x, a.ld, r, 8 * c8), a.cols - 8 * c8, a.wide);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, magnitude(x.value(i)));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(max(part[0], part[1]), max(part[2], part[3]));
  float scale, inv;
  scale_of(__uint_as_float(m), scale, inv);
  if (threadIdx.x == 0) a.row_scale[r] = scale;
  for (uint32_t c8 = threadIdx.x; c8 < c8s; c8 += 256) {
    Eight<TYPE> x;
    const uint32_t n = a.cols - 8 * c8;
    x.load(element_at<TYPE>(a.x, a.ld, r, 8 * c8), n, a.wide);
    HalfWords h = {};
    if (a.stochastic) h = draw_block(a.draws, iteration, r, c8);
    uint32_t q[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i >> 2] |= level_of(x.value(i), inv, a.stochastic, half_word(h, i)) << (8 * (i & 3));
    int8_t* out = a.q_rows + (r * a.q_rows_ld + 8 * c8);
    if (n >= 8) {
      *reinterpret_cast<uint2*>(out) = make_uint2(q[0], q[1]);
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if ((uint32_t)i < n) out[i] = (int8_t)(q[i >> 2] >> (8 * (i & 3)));
    }
  }
}

// Maxima (and sums) of a strip of 512 columns over a chunk of rows: a wavefront reads a row of the strip
// at a time.
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_column_max(QuantizeArgs a) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t c = blockIdx.x * kStripCols + 8 * lane;
  const uint32_t r0 = blockIdx.y * a.chunk_rows, r1 = min(r0 + a.chunk_rows, a.rows);
  __shared__ uint32_t maxima[4][kStripCols];
  __shared__ float sums[4][kStripCols];
  uint32_t m[8] = {};
  float s[8] = {};
  if (c < a.cols) {
    for (uint32_t r = r0 + wave; r < r1; r += 4) {
      Eight<TYPE> x;
      x.load(element_at<TYPE>(a.x, a.ld, r, c), a.cols - c, a.wide);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m[i] = max(m[i], magnitude(x.value(i)));
        s[i] += x.value(i);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) { maxima[wave][8 * lane + i] = m[i]; sums[wave][8 * lane + i] = s[i]; }
  __syncthreads();
  for (uint32_t j = threadIdx.x; j < kStripCols; j += 256) {
    const uint32_t col = blockIdx.x * kStripCols + j;
    if (col >= a.cols) continue;
    const uint64_t at = (uint64_t)blockIdx.y * a.cols + col;
    if (a.part_max) a.part_max[at] = max(max(maxima[0][j], maxima[1][j]), max(maxima[2][j], maxima[3][j]));
    if (a.part_sum) a.part_sum[at] = (sums[0][j] + sums[1][j]) + (sums[2][j] + sums[3][j]);
  }
}

// One column per thread: the chunks' maxima and sums.
__global__ __launch_bounds__(256) void k_column_scale(QuantizeArgs a) {
  const uint32_t c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  uint32_t m = 0;
  float s = 0.0f;
  for (uint32_t k = 0; k < a.chunks; ++k) {
    if (a.part_max) m = max(m, a.part_max[(uint64_t)k * a.cols + c]);
    if (a.part_sum) s += a.part_sum[(uint64_t)k * a.cols + c];
  }
  if (a.part_max) {
    float scale, inv;
    scale_of(__uint_as_float(m), scale, inv);
    a.col_max[c] = inv;
    a.col_scale[c] = scale;
  }
  if (a.part_sum) a.col_sum[c] = s;
}

// A tile of 128 rows and 64 columns: a thread quantizes 8 columns of 4 rows, whose levels of one column make
// a word in LDS; the tile leaves as 64 rows of 128 bytes.
constexpr uint32_t kTileRows = 128, kTileCols = 64;

template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_quantize_columns(QuantizeArgs a) {
  __shared__ uint32_t tile[kTileCols][kTileRows / 4 + 1];
  const uint32_t strips = (a.cols + kTileCols - 1) / kTileCols;
  const uint32_t c0 = blockIdx.x % strips * kTileCols, r0 = blockIdx.x / strips * kTileRows;
  const uint32_t c = c0 + 8 * (threadIdx.x & 7), r = r0 + 4 * (threadIdx.x >> 3);
  const uint32_t iteration = draw_iteration(a.draws);
  if (c < a.cols) {
    float inv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) inv[i] = c + i < a.cols ? a.col_max[c + i] : 0.0f;
    uint32_t q[8] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (r + j >= a.rows) break;
      Eight<TYPE> x;
      x.load(element_at<TYPE>(a.x, a.ld, r + j, c), a.cols - c, a.wide);
      HalfWords h = {};
      if (a.stochastic) h = draw_block(a.draws, iteration, r + j, c / 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] |= level_of(x.value(i), inv[i], a.stochastic, half_word(h, i)) << (8 * j);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) tile[8 * (threadIdx.x & 7) + i][threadIdx.x >> 3] = q[i];
  }
  __syncthreads();
  for (uint32_t j = threadIdx.x; j < kTileCols * (kTileRows / 4); j += 256) {
    const uint32_t col = j / (kTileRows / 4), w = j % (kTileRows / 4), row = r0 + 4 * w;
    if (c0 + col >= a.cols || row >= a.rows) continue;
    int8_t* out = a.q_cols + ((c0 + col) * a.q_cols_ld + row);
    const uint32_t v = tile[col][w], n = a.rows - row;
    if (n >= 4) *reinterpret_cast<uint32_t*>(out) = v;
    else for (uint32_t i = 0; i < n; ++i) out[i] = (int8_t)(v >> (8 * i));
  }
}

}  // namespace

void plan_columns(uint32_t rows, uint32_t cols, uint32_t& chunks, uint32_t& chunk_rows) {
  const uint32_t strips = (cols + kStripCols - 1) / kStripCols;
  const uint32_t want = strips ? (1024 + strips - 1) / strips : 1;
  chunk_rows = rows / want < 32 ? 32 : (rows + want - 1) / want;
  chunks = (rows + chunk_rows - 1) / chunk_rows;
}

hipError_t launch_quantize_rows(const QuantizeArgs& a, uint32_t type, hipStream_t st) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.rows), dim3(256), 0, st, a); };
  if (type == QSGD_TYPE_F32) go(k_quantize_rows<QSGD_TYPE_F32>);
  else if (type == QSGD_TYPE_BF16) go(k_quantize_rows<QSGD_TYPE_BF16>);
  else go(k_quantize_rows<QSGD_TYPE_F16>);
  return hipGetLastError();
}

hipError_t launch_column_max(const QuantizeArgs& a, uint32_t type, hipStream_t st) {
  const dim3 grid((a.cols + kStripCols - 1) / kStripCols, a.chunks);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (a.chunks == 0) {}
  else if (type == QSGD_TYPE_F32) go(k_column_max<QSGD_TYPE_F32>);
  else if (type == QSGD_TYPE_BF16) go(k_column_max<QSGD_TYPE_BF16>);
  else go(k_column_max<QSGD_TYPE_F16>);
  if (const hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(k_column_scale, dim3((a.cols + 255) / 256), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_quantize_columns(const QuantizeArgs& a, uint32_t type, hipStream_t st) {
  const uint64_t tiles = (uint64_t)((a.cols + kTileCols - 1) / kTileCols) * ((a.rows + kTileRows - 1) / kTileRows);
  if (tiles == 0) return hipSuccess;
  if (tiles > 0x7FFFFFFFull) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)tiles);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (type == QSGD_TYPE_F32) go(k_quantize_columns<QSGD_TYPE_F32>);
  else if (type == QSGD_TYPE_BF16) go(k_quantize_columns<QSGD_TYPE_BF16>);
  else go(k_quantize_columns<QSGD_TYPE_F16>);
  return hipGetLastError();
}

}  // namespace qsgd
