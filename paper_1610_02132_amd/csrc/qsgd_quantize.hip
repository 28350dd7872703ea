// Quantizer Q_s of Sec. 3.1 (Eq. 2) with s = 127 and max scaling (Sec. 4), a bucket being a row or a
// column of a matrix, levels as signed bytes.  Two launches for any number of matrices: the first makes the row forms and the
// columns' largest magnitudes (and sums) over chunks of rows, the second the column forms, transposed through LDS.
// The row form reads a row once, the column form reads the matrix twice: the columns of a tall matrix do not fit a compute unit.
// (Sixteen columns of some 2000 rows of 16 bits would; such short matrices take the same two launches, and a chain of load, maximum
// and level in each is their time: both forms of 2047 x 1001 fp16 5.8 and 6.0 us.)  Rows of 8192 x 4096 bf16 to the nearest level
// are bound by memory: 19 to 21 us by the card, 4.8 to 5.2 TB/s.  With draws they take 24 to 25.5: the ten rounds of the generator for
// eight elements are as many instructions as their levels, and over 80% of the slots for vector instructions are taken.  Gradients of 8192
// tokens, 4096 -> 4096 bf16: 57 us for 256 MiB in the first launch (half of the slots; 5.7 wavefronts on a SIMD wait 65% of their time)
// and 46 us for 240 MiB in the second (95% of them or more).
#include <algorithm>

#include "qsgd_layer.hpp"
#include "qsgd_levels.hpp"

namespace qsgd {
namespace {

constexpr int kHeld = 4;   // blocks of eight columns of a row that a lane holds in registers

// Rows `first` and following, one to 256 / LANES of the workgroup's parts.
template <uint32_t TYPE, bool STOCHASTIC, int LANES>
__device__ __forceinline__ void rows_block(const QuantizeArgs& a, uint32_t first, uint32_t* shared) {
  // (the row is one for a wavefront, which the compiler is told)
  const uint32_t lane = threadIdx.x % LANES, r = __builtin_amdgcn_readfirstlane(first + threadIdx.x / LANES), c8s = (a.cols + 7) / 8;
  const bool have = r < a.rows;
  Eight<TYPE> held[kHeld];
  Largest<TYPE> most;
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const uint32_t c8 = u * LANES + lane;
    if (have && c8 < c8s) {
      held[u].load(element_at<TYPE>(a.x, a.ld, r, 8 * c8), a.cols - 8 * c8);
      most.add(held[u]);
    }
  }
  for (uint32_t c8 = kHeld * LANES + lane; have && c8 < c8s; c8 += LANES) {
    Eight<TYPE> x;
    x.load(element_at<TYPE>(a.x, a.ld, r, 8 * c8), a.cols - 8 * c8);
    most.add(x);
  }
  HalfWords draws[kHeld] = {};   // of the blocks held, while these are on their way
  const uint32_t iteration = STOCHASTIC ? draw_iteration(a.draws) : 0;
  if constexpr (STOCHASTIC) {
    static_assert(kHeld == 4, "");
    draw_blocks<2>(a.draws, iteration, {r, r}, {lane, LANES + lane}, draws);
    if (c8s > 2 * LANES) draw_blocks<2>(a.draws, iteration, {r, r}, {2 * LANES + lane, 3 * LANES + lane}, draws + 2);
  }
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, most.column(i));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(shared[0], shared[1]), max(shared[2], shared[3]));
  }
  if (!have) return;
  float scale, inv;
  scale_of(__uint_as_float(m), scale, inv);
  if (lane == 0) a.row_scale[r] = scale;
  auto put = [&](const Eight<TYPE>& x, uint32_t c8, const HalfWords& h) {
    uint32_t q[2];
    eight_levels<TYPE, STOCHASTIC>(x, inv, h, q);
    int8_t* out = a.q_rows + (r * a.q_rows_ld + 8 * c8);
    const uint32_t n = a.cols - 8 * c8;
    if (n >= 8) {
      *reinterpret_cast<uint2*>(out) = make_uint2(q[0], q[1]);
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if ((uint32_t)i < n) out[i] = (int8_t)(q[i >> 2] >> (8 * (i & 3)));
    }
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const uint32_t c8 = u * LANES + lane;
    if (c8 < c8s) put(held[u], c8, draws[u]);
  }
  for (uint32_t c8 = kHeld * LANES + lane; c8 < c8s; c8 += LANES) {
    Eight<TYPE> x;
    x.load(element_at<TYPE>(a.x, a.ld, r, 8 * c8), a.cols - 8 * c8);
    HalfWords h = {};
    if constexpr (STOCHASTIC) h = draw_block(a.draws, iteration, r, c8);
    put(x, c8, h);
  }
}

// The place of a workgroup among a matrix's strips, strip by strip and then down.  Where rows do not start at lines, strips share
// lines: neighbours then run on one XCD (equal numbers modulo 8), whose L2 has them (columns of 5377 x 3393 fp16 35.1 -> 27.9 us,
// both forms of 2047 x 1001 12.0 -> 11.3; rows of whole lines are faster spread over all: both forms of 8192 x 4096 bf16 48.5, 52.4).
__device__ __forceinline__ uint32_t placed(const QuantizeArgs& a, uint32_t block, uint32_t blocks) {
  const uint32_t xcd = block % 8;
  return a.shared_lines ? xcd * (blocks / 8) + min(xcd, blocks % 8) + block / 8 : block;
}

// Maxima (and sums) of 8 * a.strip_lanes columns over a chunk of rows; strip_lanes lanes read a row of them.
template <uint32_t TYPE>
__device__ __forceinline__ void columns_block(const QuantizeArgs& a, uint32_t block, uint32_t* shared) {
  const uint32_t lanes = a.strip_lanes, strips = (a.cols + 8 * lanes - 1) / (8 * lanes);
  const uint32_t lane = threadIdx.x % lanes, part = threadIdx.x / lanes, parts = 256 / lanes;
  block = placed(a, block, a.max_blocks);
  const uint32_t strip = block % strips, chunk = block / strips, c = 8 * (strip * lanes + lane);
  const uint32_t r0 = chunk * a.chunk_rows, r1 = min(r0 + a.chunk_rows, a.rows);
  Largest<TYPE> most;
  float s[8] = {};
  const bool sums = a.part_sum != nullptr;
  if (c < a.cols) {
    auto take = [&](const Eight<TYPE>& x) {
      most.add(x);
      if (sums) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += x.value(i);
      }
    };
    uint32_t r = r0 + part;
    for (; r + 3 * parts < r1; r += 4 * parts) {   // (four rows on their way)
      Eight<TYPE> x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u].load(element_at<TYPE>(a.x, a.ld, r + u * parts, c), a.cols - c);
#pragma unroll
      for (int u = 0; u < 4; ++u) take(x[u]);
    }
    for (; r < r1; r += parts) {
      Eight<TYPE> x;
      x.load(element_at<TYPE>(a.x, a.ld, r, c), a.cols - c);
      take(x);
    }
  }
  // the parts' results: eight of them to a thread, then what is left to one per column
  const uint32_t width = 8 * lanes;
  uint32_t* const most_of = shared;
  float* const sum_of = reinterpret_cast<float*>(shared + 256 * 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    most_of[width * part + 8 * lane + i] = most.column(i);
    if (sums) sum_of[width * part + 8 * lane + i] = s[i];
  }
  __syncthreads();
  const uint32_t col = threadIdx.x % width, piece = threadIdx.x / width;
  uint32_t m = 0;
  float sum = 0.0f;
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    m = max(m, most_of[width * (8 * piece + i) + col]);
    if (sums) sum += sum_of[width * (8 * piece + i) + col];
  }
  __syncthreads();
  most_of[threadIdx.x] = m;
  if (sums) sum_of[threadIdx.x] = sum;
  __syncthreads();
  const uint32_t to_c = width * strip + threadIdx.x;
  if (threadIdx.x < width && to_c < a.cols) {
    for (uint32_t i = 1; i < 256 / width; ++i) {
      m = max(m, most_of[width * i + threadIdx.x]);
      if (sums) sum += sum_of[width * i + threadIdx.x];
    }
    const uint64_t to = (uint64_t)chunk * a.cols + to_c;
    if (a.part_max) a.part_max[to] = m;
    if (sums) a.part_sum[to] = sum;
  }
}

// The longer workgroups, a column strip's, come first: those of single rows fill in behind them (both forms of 8192 x 4096
// bf16, stochastic, the whole call: 51.6 us, rows first 55.0; fp32 74.9 and 82.1).
template <uint32_t TYPE, bool STOCHASTIC>
__global__ __launch_bounds__(256) void k_quantize_rows(QuantizeJobs jobs) {
  __shared__ uint32_t shared[2 * 256 * 8];
  uint32_t block = blockIdx.x;
  for (uint32_t j = 0; j < jobs.count; ++j) {
    const QuantizeArgs& a = jobs.job[j];
    if (block < a.max_blocks) return columns_block<TYPE>(a, block, shared);
    block -= a.max_blocks;
    if (block < a.row_blocks) {
      if (a.row_lanes == 64) rows_block<TYPE, STOCHASTIC, 64>(a, 4 * block, shared);
      else rows_block<TYPE, STOCHASTIC, 256>(a, block, shared);
      return;
    }
    block -= a.row_blocks;
  }
}

// The column form of 64 columns and up to 512 rows, 128 rows at a time: a thread quantizes 8 columns of 4 rows, whose
// levels of one column make a word in LDS; 16 bytes of a column's 128 leave with a lane.
template <uint32_t TYPE, bool STOCHASTIC>
__global__ __launch_bounds__(256) void k_quantize_columns(QuantizeJobs jobs) {
  __shared__ __attribute__((aligned(16))) uint32_t tiles[2][64 * 32];   // in turn, with one wait between them
  __shared__ uint32_t found[4][64];
  __shared__ float added[4][64], factor[64];
  uint32_t block = blockIdx.x, j = 0;
  while (block >= jobs.job[j].tile_blocks) block -= jobs.job[j++].tile_blocks;   // (the grid is their sum)
  const QuantizeArgs& a = jobs.job[j];
  block = placed(a, block, a.tile_blocks);
  const uint32_t strips = (a.cols + 63) / 64, c0 = block % strips * 64, first = block / strips * a.tile_rows;
  const uint32_t cx = threadIdx.x & 7, ry = threadIdx.x >> 3, c = c0 + 8 * cx;
  const uint32_t iteration = STOCHASTIC ? draw_iteration(a.draws) : 0;
  const uint32_t end = min(first + a.tile_rows, a.rows);
  Eight<TYPE> x[4];
  HalfWords h[4];
  const uint32_t left = c < a.cols ? a.cols - c : 0;
  auto load = [&](uint32_t r0) {   // eight columns of four of 128 rows, and their draws; the last row again for those behind it
    using bits = typename Element<TYPE>::bits;
    const uint32_t r = r0 + 4 * ry;
    const bits* p[4] = {reinterpret_cast<const bits*>(a.x) + (min(r, end - 1) * a.ld + c)};
    if (r0 + 128 <= end) {
#pragma unroll
      for (int i = 1; i < 4; ++i) p[i] = p[0] + i * a.ld;
    } else {
#pragma unroll
      for (int i = 1; i < 4; ++i) p[i] = p[i - 1] + (r + i < end ? a.ld : 0);
    }
    if (left >= 8) {
      if (a.stream) {
        asm volatile("");   // (the two ways are not to be made one)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].template load<true>(p[i], 8);
        asm volatile("");
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load(p[i], 8);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = {};
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if ((uint32_t)e < left) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i].set(e, p[i][e]);
        }
    }
    if constexpr (STOCHASTIC) draw_blocks<4>(a.draws, iteration, {r, r + 1, r + 2, r + 3}, {c / 8, c / 8, c / 8, c / 8}, h);
  };
  if (a.part_max && first < end) load(first);
  {   // the chunks' maxima and sums, by four threads to a column
    const uint32_t column = c0 + (threadIdx.x & 63), part = threadIdx.x >> 6;
    uint32_t m = 0;
    float s = 0.0f;
    const bool sums = a.part_sum && first == 0;
    if (column < a.cols) {
      for (uint32_t k = part; k < a.chunks; k += 16) {   // (four on their way)
        uint32_t v[4] = {};
        float w[4] = {};
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
          const uint64_t at = (uint64_t)(k + 4 * i) * a.cols + column;
          if (k + 4 * i < a.chunks) {
            if (a.part_max) v[i] = a.part_max[at];
            if (sums) w[i] = a.part_sum[at];
          }
        }
        m = max(m, max(max(v[0], v[1]), max(v[2], v[3])));
        s += (w[0] + w[1]) + (w[2] + w[3]);
      }
    }
    found[part][threadIdx.x & 63] = m;
    added[part][threadIdx.x & 63] = s;
    __syncthreads();
    if (threadIdx.x < 64) {
      const uint32_t t = threadIdx.x;
      m = max(max(found[0][t], found[1][t]), max(found[2][t], found[3][t]));
      float scale, inv;
      scale_of(__uint_as_float(m), scale, inv);
      factor[t] = inv;
      if (first == 0 && column < a.cols) {
        if (a.part_max) a.col_scale[column] = scale;
        if (sums) a.col_sum[column] = (added[0][t] + added[1][t]) + (added[2][t] + added[3][t]);
      }
    }
    __syncthreads();
  }
  if (!a.part_max) return;
  float inv[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) inv[i] = factor[8 * cx + i];
  // word w of column n: the 16-byte places of a column change with its number, so that eight threads' words do not meet
  auto at = [&](uint32_t n, uint32_t w) { return 32 * n + 4 * ((w >> 2) ^ (n >> 3 & 7)) + (w & 3); };
  for (uint32_t r0 = first, turn = 0; r0 < end; r0 += 128, turn ^= 1) {
    uint32_t* const tile = tiles[turn];
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      float t[4];
      uint32_t draw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        t[i] = x[i].value(n) * (STOCHASTIC ? -inv[n] : inv[n]);
        draw[i] = STOCHASTIC ? half_word(h[i], n) : 0;
      }
      tile[at(8 * cx + n, ry)] = STOCHASTIC ? stochastic_levels(t, draw) : nearest_levels(t);
    }
    if (r0 + 128 < end) load(r0 + 128);
    __syncthreads();
#pragma unroll
    for (uint32_t p = 0; p < 2; ++p) {
      const uint32_t n = 32 * p + threadIdx.x / 8, row = r0 + 16 * (threadIdx.x & 7);
      if (c0 + n < a.cols && row < a.rows) {
        const uint4 v = *reinterpret_cast<const uint4*>(&tile[at(n, 4 * (threadIdx.x & 7))]);
        int8_t* out = a.q_cols + ((c0 + n) * a.q_cols_ld + row);
        if (a.rows - row >= 16) {
          *reinterpret_cast<uint4*>(out) = v;
        } else {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (uint32_t i = 0; i < 15; ++i)
            if (row + i < a.rows) out[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
        }
      }
    }
  }
}

}  // namespace

void plan_columns(uint32_t rows, uint32_t cols, uint32_t& strip_lanes, uint32_t& chunks, uint32_t& chunk_rows) {
  strip_lanes = 16;
  while (strip_lanes > 1 && 4 * strip_lanes >= cols) strip_lanes /= 2;   // narrow matrices: more rows side by side
  const uint64_t strips = (cols + 8ull * strip_lanes - 1) / (8 * strip_lanes);
  // about 512 workgroups, 64 chunks at most (each is read again by every tile of the second launch), and four rows
  // at least to every thread
  const uint64_t want = strips ? (512 + strips - 1) / strips : 1;
  const uint64_t least = 4ull * (256 / strip_lanes);
  const uint64_t each = (rows + (want < 64 ? want : 64) - 1) / (want < 64 ? want : 64);
  chunk_rows = (uint32_t)(each < least ? least : each);
  chunks = (rows + chunk_rows - 1) / chunk_rows;
}

// At most 64 chunks, of 64 rows at least, and from 1024 columns on one for each of 512 / strips, rounded up, strips of 128 columns.
uint64_t column_numbers(uint64_t rows, uint64_t cols) {
  return std::min(cols * std::min<uint64_t>((rows + 63) / 64, 64), 512 * 128 + cols);
}

uint64_t plan_quantize(QuantizeJobs& jobs, uint32_t type) {
  uint64_t first = 0, second = 0;
  for (uint32_t j = 0; j < jobs.count; ++j) {
    QuantizeArgs& a = jobs.job[j];
    const bool columns = a.part_max || a.part_sum;
    a.row_lanes = a.cols <= 8 * 64 * kHeld && a.rows >= 1024 ? 64 : 256;   // a wavefront to a row, or four
    const uint64_t rows = !a.row_scale ? 0 : a.row_lanes == 64 ? (a.rows + 3) / 4 : a.rows;
    const uint64_t maxima = columns ? (a.cols + 8 * a.strip_lanes - 1) / (8 * a.strip_lanes) * (uint64_t)a.chunks : 0;
    const uint64_t strips = (a.cols + 63) / 64;
    a.shared_lines = ((reinterpret_cast<uintptr_t>(a.x) | a.ld * (type == QSGD_TYPE_F32 ? 4 : 2)) & 127) != 0;
    // the last reading of a matrix that L2 does not hold goes past the caches (gradients of 8192 tokens, 4096 -> 4096
    // bf16: 360 us without, 347 with)
    a.stream = (uint64_t)a.rows * a.cols * (type == QSGD_TYPE_F32 ? 4 : 2) >= 32ull << 20;
    // every workgroup reads the chunks' maxima: few rows to one only where there would be too few of them
    // (2047 x 1001, both forms, the whole call: 128 rows 16.1 us, 512 rows 22.2; 8192 x 4096 the same)
    a.tile_rows = 512;
    while (a.tile_rows > 128 && strips * ((a.rows + a.tile_rows - 1) / a.tile_rows) < 1024) a.tile_rows /= 2;
    // (sums alone, and the scales of no rows, need a workgroup to a strip)
    const uint64_t tiles = !columns ? 0 : strips * (a.part_max && a.rows ? (a.rows + a.tile_rows - 1) / a.tile_rows : 1);
    a.row_blocks = (uint32_t)rows; a.max_blocks = (uint32_t)maxima; a.tile_blocks = (uint32_t)tiles;
    first += rows + maxima;
    second += tiles;
  }
  jobs.blocks[0] = (uint32_t)first; jobs.blocks[1] = (uint32_t)second;
  return first > second ? first : second;
}

hipError_t launch_quantize(const QuantizeJobs& jobs, uint32_t type, bool stochastic, hipStream_t st, bool second) {
  const uint32_t blocks = jobs.blocks[second];
  if (blocks == 0) return hipSuccess;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, jobs); };
  auto pick = [&](auto type_c) {
    constexpr uint32_t T = decltype(type_c)::value;
    if (second) stochastic ? go(k_quantize_columns<T, true>) : go(k_quantize_columns<T, false>);
    else stochastic ? go(k_quantize_rows<T, true>) : go(k_quantize_rows<T, false>);
  };
  if (type == QSGD_TYPE_F32) pick(std::integral_constant<uint32_t, QSGD_TYPE_F32>{});
  else if (type == QSGD_TYPE_BF16) pick(std::integral_constant<uint32_t, QSGD_TYPE_BF16>{});
  else pick(std::integral_constant<uint32_t, QSGD_TYPE_F16>{});
  return hipGetLastError();
}

}  // namespace qsgd
