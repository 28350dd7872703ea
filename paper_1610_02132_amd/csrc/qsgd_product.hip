// Product of 8-bit matrices with a scale per row of each:
//   y[m][n] = (sum_k a[m][k] b[n][k]) a_scale[m] b_scale[n] + bias[n],
// both operands with k contiguous.  The sum is an integer and exact whatever the order, so that pieces of k
// can be summed apart (a workspace of int32 sums, joined in 64 bits) without changing the result.
#include <algorithm>
#include <cmath>

#include "qsgd_layer.hpp"
#include "qsgd_levels.hpp"

namespace qsgd {
namespace {

using int4v = __attribute__((ext_vector_type(4))) int;
using int16v = __attribute__((ext_vector_type(16))) int;

// Most of k in one piece: 130816 * 128 * 128 < 2^31, and a multiple of 256.
constexpr uint32_t kMostK = 130816;
constexpr uint32_t kSums = 99;   // "type" of a piece's sums in the workspace

// The sum times the row's scale, times the column's, plus the bias, the last two in one rounding.  Where the row's scale is above
// kBigScale in size the first product, of a sum below 2^37, could leave fp32 although the result does not: it is taken 2^64 times
// smaller and the column's scale larger, both exactly (the product is at least 2^26 then, so that a column's scale that leaves
// fp32 on the way belongs to a result that does; a sum of nothing keeps the column's scale).
constexpr float kBigScale = 0x1p90f;
__device__ __forceinline__ float result(float sum, float s, float t, float bias) {
  const bool big = fabsf(s) > kBigScale;
  const float u = big ? sum * (s * 0x1p-64f) : sum * s;
  return __builtin_fmaf(u, big && u != 0.0f ? t * 0x1p64f : t, bias);
}

__device__ __forceinline__ void put(const ProductArgs& a, uint32_t m, uint32_t n, float sum, float row_scale) {
  const float v = result(sum, row_scale, a.b_scale[n], a.bias ? a.bias[n] : 0.0f);
  const uint64_t at = m * a.y_ld + n;
  if (a.type == QSGD_TYPE_F32) reinterpret_cast<float*>(a.y)[at] = v;
  else reinterpret_cast<uint16_t*>(a.y)[at] = (uint16_t)(a.type == QSGD_TYPE_BF16 ? Element<QSGD_TYPE_BF16>::narrow(v) : Element<QSGD_TYPE_F16>::narrow(v));
}

// 16 bytes of an operand from k on, those behind K zeroed.
__device__ __forceinline__ int4v masked(int4v v, uint32_t k, uint32_t K) {
  const uint32_t n = k < K ? K - k : 0u;   // valid bytes
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    const uint32_t have = n > 4 * j ? min(n - 4 * j, 4u) : 0u;
    v[j] = have == 4 ? v[j] : (int)((uint32_t)v[j] & ((1u << (8 * have)) - 1u));
  }
  return v;
}

// ... of its row, straight from memory; the row is clamped into the matrix (its results are not written), k into the row.
__device__ __forceinline__ int4v operand(const int8_t* p, uint64_t ld, uint32_t row, uint32_t rows, uint32_t k, uint32_t K) {
  return *reinterpret_cast<const int4v*>(p + (min(row, rows - 1) * ld + min(k, (K + 15) / 16 * 16 - 16)));
}

// ---- tiles ------------------------------------------------------------------------
// A workgroup of four wavefronts makes a tile of 64 MI x 64 NI results, each wavefront 32 MI x 32 NI of them in
// registers (MFMA 32x32x32: the weights' rows are the rows, so that a lane holds four neighbouring results of
// one row of y).  128 bytes of k, whole cache lines, are a stage; STAGES of them are in LDS, loaded straight from memory.
// Slot s of a row of 128 bytes holds chunk s ^ swizzle(row).
// 8192^3, tiles of 256: 434 to 457 us by the card = 2400 to 2530 Tops, the matrix units busy in 73% of the cycles at a clock that
// the power of these products brings down to 1.5 to 1.7 GHz (matrix instructions alone on such values: 3040 Tops).  A tile of 256
// reads half as many bytes of LDS for a matrix instruction as one of 128 (4096^3 60 to 62 us, tiles of 128 70), but small products
// do not fill the card with such tiles; those of 64 are for them, with four stages where a compute unit has no second workgroup to
// hide the loads of one (256 x 4096 x 4096 10.2 us, two stages 17.2, tiles of 128 23.1), and those of 128 x 64 in between
// (2048^3 14.4 us, tiles of 128 16.4, of 64 17.2).
constexpr uint32_t kDepth = 128;   // bytes of k in a stage

// Rows whose 16-byte chunks of one number are read together (8 or 16 neighbours, or fours of them whose numbers differ
// in bits 2 and 3) get places in different banks: by bits 1, 2 and 3 where bit 0 is equal, and by bits 0, 1 and 2.
__device__ __forceinline__ uint32_t swizzle(uint32_t row) { return (row >> 1 & 3) | ((row ^ row >> 3) & 1) << 2; }

__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t from, uint8_t* to, uint32_t voffset, uint32_t soffset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, voffset, soffset, 0, 0);
}

// Waits until at most N of this wavefront's loads are on their way, and for all its reads of LDS.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The tile of a workgroup: those that run on one XCD (workgroups i with equal i % 8) are neighbours, in bands of four
// rows of tiles, so that its L2 serves their operands.
__device__ __forceinline__ void place_tile(uint32_t id, uint32_t down, uint32_t across, uint32_t& tm, uint32_t& tn) {
  const uint32_t tiles = down * across, q = tiles / 8, r = tiles % 8, xcd = id % 8;
  const uint32_t t = xcd * q + min(xcd, r) + id / 8;
  constexpr uint32_t kBand = 4;
  const uint32_t band = t / (kBand * across), in = t % (kBand * across), high = min(kBand, down - band * kBand);
  tm = band * kBand + in % high;
  tn = in / high;
}

// The order of the instructions since the last such mark: the matrix instructions evenly between the reads of LDS
// (and the loads), a read first.
template <int MATRIX, int READS, int LOADS>
__device__ __forceinline__ void weave() {
  constexpr int kEach = MATRIX / READS > 0 ? MATRIX / READS : 1;
#pragma unroll
  for (int i = 0; i < READS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);               // reads of LDS
    if (LOADS) __builtin_amdgcn_sched_group_barrier(0x20, LOADS / READS, 0);   // loads
    __builtin_amdgcn_sched_group_barrier(0x8, kEach, 0);             // matrix instructions
  }
  __builtin_amdgcn_sched_barrier(0);
}

// A wavefront's results (32 MI rows of y from m0 on, 32 NI columns from n0 on) leave through LDS, 32 rows at a time, so that
// a store covers whole lines, and a lane's columns, with their scales, are the same for every row.
template <int MI, int NI, uint32_t ROOM, uint32_t TYPE>
__device__ __forceinline__ void leave(const ProductArgs& a, const int16v (&acc)[MI][NI], uint8_t* stage, uint32_t m0, uint32_t n0) {
  const uint32_t lane = threadIdx.x & 63;
  constexpr uint32_t kSize = TYPE == QSGD_TYPE_F32 || TYPE == kSums ? 4 : 2, kPer = 16 / kSize;   // results of 16 bytes
  constexpr uint32_t kRow = 32 * NI * 4 + 16, kChunks = 32 * NI / kPer, kRows = 64 / kChunks;      // rows that a store covers
  static_assert(32 * kRow + 32 * MI * 4 <= ROOM, "");
  float* x_scale = reinterpret_cast<float*>(stage + 32 * kRow);
  const uint32_t n = n0 + lane % kChunks * kPer;
  float w_scale[kPer], bias[kPer];
  bool big = false;   // any row's scale is
  if constexpr (TYPE != kSums) {
#pragma unroll
    for (uint32_t e = 0; e < kPer; ++e) {
      const uint32_t at = min(n + e, a.N - 1);
      w_scale[e] = a.b_scale[at];
      bias[e] = a.bias ? a.bias[at] : 0.0f;
    }
    for (uint32_t r = lane; r < 32 * MI; r += 64) {
      x_scale[r] = a.a_scale[min(m0 + r, a.M - 1)];
      big |= fabsf(x_scale[r]) > kBigScale;
    }
    big = __any(big);
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<int4v*>(stage + (lane & 31) * kRow + (32 * j + 8 * g + 4 * (lane >> 5)) * 4) =
            int4v{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    wait_loads<63>();   // (the wavefront's writes have arrived)
#pragma unroll
    for (uint32_t it = 0; it < 32 / kRows; ++it) {
      const uint32_t row = it * kRows + lane / kChunks, m = m0 + 32 * i + row;
      const int4v* from = reinterpret_cast<const int4v*>(stage + row * kRow + lane % kChunks * kPer * 4);
      uint4 out;
      if constexpr (TYPE == kSums) {
        out = __builtin_bit_cast(uint4, from[0]);
      } else {
        const float s = x_scale[32 * i + row];
        float v[kPer];
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) v[e] = __builtin_fmaf((float)from[e / 4][e % 4] * s, w_scale[e], bias[e]);
        if (big) {
#pragma unroll
          for (uint32_t e = 0; e < kPer; ++e) v[e] = result((float)from[e / 4][e % 4], s, w_scale[e], bias[e]);
        }
        if constexpr (kSize == 4) out = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        else out = make_uint4(Element<TYPE>::narrow2(v[0], v[1]), Element<TYPE>::narrow2(v[2], v[3]),
                              Element<TYPE>::narrow2(v[4], v[5]), Element<TYPE>::narrow2(v[6], v[7]));
      }
      if (m >= a.M || n >= a.N) continue;
      uint8_t* to = TYPE == kSums ? reinterpret_cast<uint8_t*>(a.part) + (((uint64_t)blockIdx.y * a.M + m) * a.N + n) * 4
                                  : reinterpret_cast<uint8_t*>(a.y) + (m * a.y_ld + n) * kSize;
      if (n + kPer <= a.N) {
        using Words = __attribute__((ext_vector_type(4), aligned(kSize))) uint32_t;   // (a row starts anywhere)
        *reinterpret_cast<Words*>(to) = Words{out.x, out.y, out.z, out.w};
      } else {
        const uint32_t w[4] = {out.x, out.y, out.z, out.w};
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) {
          if (n + e >= a.N) break;
          if constexpr (kSize == 4) reinterpret_cast<uint32_t*>(to)[e] = w[e];
          else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
        }
      }
    }
    wait_loads<63>();   // (... and its reads)
  }
}

// f(0), f(1), ... with numbers that the compiler knows.
template <uint32_t N, class F>
__device__ __forceinline__ void static_for(F f) {
  if constexpr (N > 0) {
    static_for<N - 1>(f);
    f(std::integral_constant<uint32_t, N - 1>{});
  }
}

template <int MI, int NI, int STAGES>
__global__ __launch_bounds__(256, MI * NI > 4 ? 1 : 2) void k_product(ProductPair pair) {
  constexpr uint32_t TM = 64 * MI, TN = 64 * NI, kStage = (TM + TN) * kDepth;
  constexpr int kLoads = 2 * (MI + NI);   // of a wavefront and stage, 8 rows each
  __shared__ __attribute__((aligned(16))) uint8_t s0[kStage], s1[kStage];
  // (each stage an array of its own: the compiler then waits for none but the one that is read)
  __shared__ __attribute__((aligned(16))) uint8_t s2[STAGES > 2 ? kStage : 16], s3[STAGES > 2 ? kStage : 16];
  auto place = [&](uint32_t i) -> uint8_t* { return i == 0 ? s0 : i == 1 ? s1 : i == 2 ? s2 : s3; };
  const bool second = blockIdx.x >= pair.first;   // (of two products: the workgroups behind the first one's)
  const ProductArgs& a = pair.of[second];
  uint32_t tm, tn;
  place_tile(blockIdx.x - (second ? pair.first : 0), (a.M + TM - 1) / TM, (a.N + TN - 1) / TN, tm, tn);
  const uint32_t m0 = tm * TM, n0 = tn * TN;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t k0 = blockIdx.y * a.split_k, k1 = min(k0 + a.split_k, a.K);
  // stages, and those of them that k fills; the last may be a part
  const uint32_t steps = (k1 - k0 + kDepth - 1) / kDepth, whole = (k1 - k0) / kDepth;
  const uint32_t rows_a = min(TM, a.M - m0), rows_b = min(TN, a.N - n0), padded = (a.K + 15) / 16 * 16;
  const auto from_a = __builtin_amdgcn_make_buffer_rsrc((void*)(a.a + m0 * a.a_ld), 0, (int)((rows_a - 1) * (uint32_t)a.a_ld + padded), 0x27000);
  const auto from_b = __builtin_amdgcn_make_buffer_rsrc((void*)(a.b + n0 * a.b_ld), 0, (int)((rows_b - 1) * (uint32_t)a.b_ld + padded), 0x27000);
  uint32_t at_a[2 * MI], at_b[2 * NI];   // rows are clamped into the matrix
  auto chunk = [&](int i) { return 16 * ((lane & 7) ^ swizzle((lane >> 3) + 8 * (i & 1))); };
#pragma unroll
  for (int i = 0; i < 2 * MI; ++i) at_a[i] = min(8u * (2 * MI * wave + i) + (lane >> 3), rows_a - 1) * (uint32_t)a.a_ld + chunk(i);
#pragma unroll
  for (int i = 0; i < 2 * NI; ++i) at_b[i] = min(8u * (2 * NI * wave + i) + (lane >> 3), rows_b - 1) * (uint32_t)a.b_ld + chunk(i);
  // Loads [from, to) of a stage; the last stage may be a part, whose chunks are clamped into the row.
  auto load = [&](uint32_t step, uint8_t* place, int from, int to, bool last) {
    const uint32_t k = k0 + step * kDepth, end = padded - 16 - k;
    auto clamped = [&](uint32_t at, int i) { return last && step >= whole ? at - chunk(i) + min(chunk(i), end) : at; };
#pragma unroll
    for (int i = 0; i < 2 * MI; ++i)
      if (i >= from && i < to) load_to_lds(from_a, place + 1024 * (2 * MI * wave + i), clamped(at_a[i], i), k);
#pragma unroll
    for (int i = 0; i < 2 * NI; ++i)
      if (2 * MI + i >= from && 2 * MI + i < to)
        load_to_lds(from_b, place + TM * kDepth + 1024 * (2 * NI * wave + i), clamped(at_b[i], i), k);
  };
  const uint32_t wm = (wave & 1) * 32 * MI, wn = (wave >> 1) * 32 * NI;   // the wavefront's part of the tile
  const uint32_t frag = (lane & 31) * kDepth + 16 * ((lane >> 5) ^ swizzle(lane));
  int4v xf[2][MI], wf[2][NI];
  auto read = [&](const uint8_t* from, int quarter) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      wf[quarter & 1][i] = *reinterpret_cast<const int4v*>(from + (TM + wn + 32 * i) * kDepth + (frag ^ (32 * quarter)));
#pragma unroll
    for (int i = 0; i < MI; ++i)
      xf[quarter & 1][i] = *reinterpret_cast<const int4v*>(from + (wm + 32 * i) * kDepth + (frag ^ (32 * quarter)));
  };
  int16v acc[MI][NI] = {};
  auto multiply = [&](int quarter) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[quarter & 1][j], xf[quarter & 1][i], acc[i][j], 0, 0, 0);
  };
  if constexpr (STAGES == 2) {
    // Stage `now` has its first quarter in registers when its step begins.  Behind the barrier all wavefronts have read
    // the stage and hold the next one's loads: its place is loaded again, one part of the loads with the last quarter and
    // one with the next step's first, as they come faster than they are taken.
    constexpr int kPart = kLoads / 2;
    auto step = [&](uint8_t* now, uint8_t* other, uint32_t s) {
      load(s + 1, other, kPart, kLoads, false);
      read(now, 1);
      multiply(0);
      weave<MI * NI, MI + NI, (kLoads - kPart)>();
      read(now, 2);
      multiply(1);
      weave<MI * NI, MI + NI, 0>();
      read(now, 3);
      multiply(2);
      weave<MI * NI, MI + NI, 0>();
      wait_loads<0>();
      meet();
      load(s + 2, now, 0, kPart, false);
      read(other, 0);
      multiply(3);
      weave<MI * NI, MI + NI, kPart>();
    };
    auto last_step = [&](uint8_t* now, uint8_t* other, uint32_t s) {   // ... of the last ones, where loads end
      if (s + 1 < steps) load(s + 1, other, kPart, kLoads, true);
      read(now, 1);
      multiply(0);
      weave<MI * NI, MI + NI, 0>();
      read(now, 2);
      multiply(1);
      weave<MI * NI, MI + NI, 0>();
      read(now, 3);
      multiply(2);
      weave<MI * NI, MI + NI, 0>();
      wait_loads<0>();
      meet();
      if (s + 2 < steps) load(s + 2, now, 0, kPart, true);
      read(other, 0);
      multiply(3);
    };
    if (steps > 0) {
      load(0, s0, 0, kLoads, true);
      if (steps > 1) { load(1, s1, 0, kPart, true); wait_loads<kPart>(); }
      else wait_loads<0>();
      meet();
      read(s0, 0);
      uint32_t s = 0;
      for (; s + 4 <= whole; s += 2) {
        step(s0, s1, s);
        step(s1, s0, s + 1);
      }
      for (; s < whole; s += 2) {
        last_step(s0, s1, s);
        if (s + 1 < whole) last_step(s1, s0, s + 1);
      }
    }
  } else {
    // The next stage is read whole while one is multiplied (333 x 1111 x 2223, all on one card: 8.2 us, a quarter ahead 8.6, eight
    // stages 9.4; on other cards up to 9.2).  A stage takes 400 clocks for 16 load instructions of 1 KiB; half as many reads of LDS
    // (every wavefront a quarter of k for the whole tile) or loads that read nothing for rows behind the matrix do not shorten it.
    static_assert(MI * NI == 1 && STAGES == 4, "");
    int4v xs[2][4], ws[2][4];
    auto read_stage = [&](const uint8_t* from, int to) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        ws[to][q] = *reinterpret_cast<const int4v*>(from + (TM + wn) * kDepth + (frag ^ (32 * q)));
        xs[to][q] = *reinterpret_cast<const int4v*>(from + wm * kDepth + (frag ^ (32 * q)));
      }
    };
    // Waits for all loads but those of the last n stages, n at most MOST.
    auto wait_stages = [&](auto most, uint32_t n) {
      static_for<decltype(most)::value + 1>([&](auto i) {
        if (n == i || (i == decltype(most)::value && n > i)) wait_loads<decltype(i)::value * kLoads>();
      });
    };
    auto step = [&](uint8_t* now, const uint8_t* next, uint32_t s, int held, bool last) {
      if (!last) wait_loads<(STAGES - 2) * kLoads>();
      else wait_stages(std::integral_constant<uint32_t, STAGES - 2>{}, s + 2 < steps ? steps - s - 2 : 0);
      meet();   // all wavefronts have read stage `now` and hold the next one's loads
      if (!last || s + STAGES < steps) load(s + STAGES, now, 0, kLoads, last);
      read_stage(next, held ^ 1);
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[0][0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(ws[held][q], xs[held][q], acc[0][0], 0, 0, 0);
      if (!last) {
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);      // reads of LDS, loads, matrix instructions
        __builtin_amdgcn_sched_group_barrier(0x20, kLoads, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, 4, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    if (steps > 0) {
      static_for<STAGES>([&](auto i) { if (i < steps) load(i, place(i), 0, kLoads, true); });
      wait_stages(std::integral_constant<uint32_t, STAGES - 1>{}, steps - 1);
      meet();
      read_stage(s0, 0);
      uint32_t s = 0;
      for (; s + 2 * STAGES <= whole; s += STAGES)
        static_for<STAGES>([&](auto i) { step(place(i), place((i + 1) % STAGES), s + i, i % 2, false); });
      for (; s < whole; s += STAGES)
        static_for<STAGES>([&](auto i) { if (s + i < whole) step(place(i), place((i + 1) % STAGES), s + i, i % 2, true); });
    }
  }
  if (steps > 0) {
    if (whole < steps) {   // the part: what lies behind K counts as zero in one of the operands
      const uint8_t* now = place(whole % STAGES);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        read(now, q);
        const uint32_t k = k0 + whole * kDepth + 32 * q + 16 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < MI; ++i) xf[q & 1][i] = masked(xf[q & 1][i], k, a.K);
        multiply(q);
      }
    }
  }
  wait_loads<0>();
  meet();   // (all wavefronts have read their last stage)
  // a wavefront's rows of y's tile, written as y's type asks
  uint8_t* stage = (wave < 2 ? s0 : s1) + (wave & 1) * (kStage / 2);
  if (a.part) leave<MI, NI, kStage / 2, kSums>(a, acc, stage, m0 + wm, n0 + wn);
  else if (a.type == QSGD_TYPE_F32) leave<MI, NI, kStage / 2, QSGD_TYPE_F32>(a, acc, stage, m0 + wm, n0 + wn);
  else if (a.type == QSGD_TYPE_BF16) leave<MI, NI, kStage / 2, QSGD_TYPE_BF16>(a, acc, stage, m0 + wm, n0 + wn);
  else leave<MI, NI, kStage / 2, QSGD_TYPE_F16>(a, acc, stage, m0 + wm, n0 + wn);
}

// ---- shallow ----------------------------------------------------------------------
// Little depth and many results: the results' bytes are what it takes.  Every wavefront makes 32 x 64 of them by itself,
// operands straight from memory (neighbours share them in the caches), so that nothing waits for a stage and 16
// wavefronts of a compute unit are at different points of theirs.  8192 x 8192 x 64: fp32 51.2 us = 5.3 TB/s, bound by
// the results' bytes; bf16 41.3 = 3.3, bound by the chain of loads, LDS and stores: 3.6 wavefronts on a SIMD wait 63% of their time.
constexpr uint32_t kShallowRows = 64, kShallowCols = 128;   // of a workgroup
constexpr uint32_t kShallowDepth = 64;                      // most of k: two matrix instructions

__global__ __launch_bounds__(256) void k_product_shallow(ProductPair pair) {
  constexpr uint32_t kRoom = 32 * (64 * 4 + 16) + 32 * 4;
  __shared__ __attribute__((aligned(16))) uint8_t staged[4][kRoom];
  const bool second = blockIdx.x >= pair.first;
  const ProductArgs& a = pair.of[second];
  uint32_t tm, tn;
  place_tile(blockIdx.x - (second ? pair.first : 0), (a.M + kShallowRows - 1) / kShallowRows, (a.N + kShallowCols - 1) / kShallowCols, tm, tn);
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t m0 = tm * kShallowRows + (wave & 1) * 32, n0 = tn * kShallowCols + (wave >> 1) * 64;
  const uint32_t row = lane & 31, own = 16 * (lane >> 5);
  int16v acc[1][2] = {};
  if (a.K > 0) {
    int4v x[2], w[2][2];
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      x[q] = operand(a.a, a.a_ld, m0 + row, a.M, 32 * q + own, a.K);
      w[q][0] = operand(a.b, a.b_ld, n0 + row, a.N, 32 * q + own, a.K);
      w[q][1] = operand(a.b, a.b_ld, n0 + 32 + row, a.N, 32 * q + own, a.K);
    }
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      if (32 * q + 32 > a.K) x[q] = masked(x[q], 32 * q + own, a.K);
      acc[0][0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[q][0], x[q], acc[0][0], 0, 0, 0);
      acc[0][1] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[q][1], x[q], acc[0][1], 0, 0, 0);
    }
  }
  if (a.type == QSGD_TYPE_F32) leave<1, 2, kRoom, QSGD_TYPE_F32>(a, acc, staged[wave], m0, n0);
  else if (a.type == QSGD_TYPE_BF16) leave<1, 2, kRoom, QSGD_TYPE_BF16>(a, acc, staged[wave], m0, n0);
  else leave<1, 2, kRoom, QSGD_TYPE_F16>(a, acc, staged[wave], m0, n0);
}

// ---- few rows ---------------------------------------------------------------------
// At most 32 rows of a: the weights' bytes are what it takes.  A workgroup has 16 of their rows and up to eight wavefronts,
// which take turns at 256 bytes of k, loaded whole into a wavefront's own piece of LDS and read from there as the matrix
// instruction wants them (a lane has 64 bytes in a row: the order of k is the same for both operands, so it need not be
// the instruction's own).  1 x 28672 x 8192 40.2 us = 5.9 TB/s, the rate of a copy; loads straight into registers, whose lanes are
// in 16 rows, 42.0; 16 wavefronts 40.9.
constexpr uint32_t kFewDepth = 256, kFewWaves = 8;

template <int MT>
__global__ __launch_bounds__(64 * kFewWaves) void k_product_few(ProductArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t staged[];   // 4 KiB for each wavefront
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const uint32_t n0 = blockIdx.x * 16, k0 = blockIdx.y * a.split_k, k1 = min(k0 + a.split_k, a.K);
  const uint32_t own = 64 * (lane >> 4), rows = min(16u, a.N - n0), padded = (a.K + 15) / 16 * 16;
  uint8_t* const place = staged + 4096 * wave;
  const auto from = __builtin_amdgcn_make_buffer_rsrc((void*)(a.b + n0 * a.b_ld), 0, (int)((rows - 1) * (uint32_t)a.b_ld + padded), 0x27000);
  // load j of a turn: rows 4 j to 4 j + 3, 256 bytes of each in a row; place s of a row holds chunk s ^ ((row - 4) % 16), so that
  // neither 16 neighbours nor fours of them from two halves of 32 lanes read one bank
  uint32_t row_at[4], chunk[4];
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    const uint32_t r = 4 * j + (lane >> 4);
    row_at[j] = min(r, rows - 1) * (uint32_t)a.b_ld;
    chunk[j] = 16 * ((lane & 15) ^ ((r - 4) & 15));
  }
  int4v acc[MT] = {};
  for (uint32_t k = k0 + wave * kFewDepth; k < k1; k += waves * kFewDepth) {
    int4v x[MT][4];
    const bool whole = k + kFewDepth <= k1;
    const uint32_t end = padded - 16 - k;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) load_to_lds(from, place + 1024 * j, row_at[j] + (whole ? chunk[j] : min(chunk[j], end)), k);
    if (whole) {
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const int8_t* p = a.a + (min(16 * t + (lane & 15), a.M - 1) * a.a_ld + k + own);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[t][j] = reinterpret_cast<const int4v*>(p)[j];
      }
    } else {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[t][j] = masked(operand(a.a, a.a_ld, 16 * t + (lane & 15), a.M, k + own + 16 * j, a.K), k + own + 16 * j, a.K);
    }
    wait_loads<0>();
    int4v w[4];
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
      w[j] = *reinterpret_cast<const int4v*>(place + 256 * (lane & 15) + 16 * ((4 * (lane >> 4) + j) ^ ((lane - 4) & 15)));
    wait_loads<63>();   // (read before the next turn's come)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[t][j], acc[t], 0, 0, 0);
  }
  int* const sums = reinterpret_cast<int*>(staged);
#pragma unroll
  for (int t = 0; t < MT; ++t)
    *reinterpret_cast<int4v*>(&sums[1024 * wave + (16 * t + (lane & 15)) * 16 + 4 * (lane >> 4)]) = acc[t];
  __syncthreads();
  for (uint32_t o = threadIdx.x; o < MT * 256; o += blockDim.x) {
    const uint32_t m = o / 16, n = n0 + o % 16;
    if (m >= a.M || n >= a.N) continue;
    int sum = 0;
    for (uint32_t s = 0; s < waves; ++s) sum += sums[1024 * s + o];
    if (a.part) a.part[((uint64_t)blockIdx.y * a.M + m) * a.N + n] = sum;
    else put(a, m, n, (float)sum, a.a_scale[m]);
  }
}

// The layer for few tokens, their quantizing included: every workgroup makes the levels of all of them (in LDS, where
// its wavefronts' turns find them) while the weights of its first turn are on their way, which costs less than a launch
// (1 x 8192 x 8192 15.2 us, 4.4 TB/s; two launches 17.2).  Bound by the chain from the tokens' maxima to the last product.
template <uint32_t TYPE, bool STOCHASTIC>
__global__ __launch_bounds__(1024) void k_linear_few(LinearArgs l) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  __shared__ uint32_t most[16];
  __shared__ float scale[16], factor[16];
  const ProductArgs& a = l.product;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  int* const sums = reinterpret_cast<int*>(lds);                       // 256 for each wavefront
  uint8_t* const levels = lds + 1024 * waves;                          // rows of `stride`, zeros behind K
  const uint32_t n0 = blockIdx.x * 16, own = 64 * (lane >> 4), whole = (a.K + kFewDepth - 1) / kFewDepth * kFewDepth;
  const uint32_t stride = whole + 16;
  int4v w[4];
  auto weights = [&](uint32_t k) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = operand(a.b, a.b_ld, n0 + (lane & 15), a.N, k + own + 16 * j, a.K);
  };
  weights(wave * kFewDepth);
  // a row to `parts` wavefronts, or several rows to one
  const uint32_t parts = waves > a.M ? waves / a.M : 1, part = wave / a.M, step = waves > a.M ? a.M : waves;
  const uint32_t row0 = part < parts ? wave % a.M : a.M, c8s = (a.K + 7) / 8;
  if (threadIdx.x < 16) most[threadIdx.x] = 0;
  __syncthreads();
  for (uint32_t m = row0; m < a.M; m += step) {
    Largest<TYPE> largest;
    for (uint32_t c8 = 64 * part + lane; c8 < c8s; c8 += 64 * parts) {
      Eight<TYPE> x;
      x.load(element_at<TYPE>(l.x, l.x_ld, m, 8 * c8), a.K - 8 * c8);
      largest.add(x);
    }
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) v = max(v, largest.column(i));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
    if (lane == 0) atomicMax(&most[m], v);
  }
  __syncthreads();
  if (threadIdx.x < a.M) scale_of(__uint_as_float(most[threadIdx.x]), scale[threadIdx.x], factor[threadIdx.x]);
  __syncthreads();
  const uint32_t iteration = STOCHASTIC ? draw_iteration(l.draws) : 0;
  for (uint32_t m = row0; m < a.M; m += step) {
    const float inv = factor[m];
    for (uint32_t c8 = 64 * part + lane; c8 < whole / 8; c8 += 64 * parts) {
      uint32_t q[2] = {0, 0};
      if (c8 < c8s) {
        Eight<TYPE> x;
        x.load(element_at<TYPE>(l.x, l.x_ld, m, 8 * c8), a.K - 8 * c8);
        HalfWords h = {};
        if constexpr (STOCHASTIC) h = draw_block(l.draws, iteration, m, c8);
        eight_levels<TYPE, STOCHASTIC>(x, inv, h, q);
      }
      *reinterpret_cast<uint2*>(levels + m * stride + 8 * c8) = make_uint2(q[0], q[1]);
    }
  }
  __syncthreads();
  int4v acc = {};
  for (uint32_t k = wave * kFewDepth; k < a.K; k += waves * kFewDepth) {
    if (k >= waves * kFewDepth) weights(k);
    const int4v* x = reinterpret_cast<const int4v*>(levels + min(lane & 15, a.M - 1) * stride + k + own);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[j], acc, 0, 0, 0);
  }
  *reinterpret_cast<int4v*>(&sums[256 * wave + (lane & 15) * 16 + 4 * (lane >> 4)]) = acc;
  __syncthreads();
  if (threadIdx.x < 256) {
    const uint32_t m = threadIdx.x / 16, n = n0 + threadIdx.x % 16;
    if (m < a.M && n < a.N) {
      int sum = 0;
      for (uint32_t s = 0; s < waves; ++s) sum += sums[256 * s + threadIdx.x];
      put(a, m, n, (float)sum, scale[m]);
    }
  }
}

// The pieces' sums, added in 64 bits: PER neighbouring results of a row to a thread, and others behind them where there
// are more than a launch counts.  Memory bound; mostly a launch (1500 x 1500 in two pieces 5 us with it).
constexpr uint32_t kMostJoinBlocks = 1u << 16;
template <int PER>
__global__ __launch_bounds__(256) void k_product_join(ProductArgs a) {
  const uint64_t all = (uint64_t)a.M * a.N;
  for (uint64_t i = PER * ((uint64_t)blockIdx.x * 256 + threadIdx.x); i < all; i += PER * 256ull * gridDim.x) {
    int64_t sum[PER] = {};
    for (uint32_t s = 0; s < a.splits; ++s) {
      int v[PER];
      if constexpr (PER == 4) *reinterpret_cast<int4v*>(v) = *reinterpret_cast<const int4v*>(a.part + s * all + i);
      else v[0] = a.part[s * all + i];
#pragma unroll
      for (int e = 0; e < PER; ++e) sum[e] += v[e];
    }
    const uint32_t m = all >> 32 ? (uint32_t)(i / a.N) : (uint32_t)i / a.N, n = (uint32_t)(i - (uint64_t)m * a.N);
#pragma unroll
    for (int e = 0; e < PER; ++e) put(a, m, n + e, (float)sum[e], a.a_scale[m]);
  }
}

}  // namespace

// Limits of pieces that are made for speed, beyond the fewest that k needs, so that product_space can say what any smaller product
// takes.  Of 500000 products the rest of the estimate would take two outside them, both of 4096 of k, which are faster in one
// (416 x 2 x 4096 8.7 us, in four pieces 9.1); 2^24 sums are those of 256 tiles of 256.
constexpr uint32_t kLeastK = 4096, kLeastPiece = 1024, kMorePieces = 16;
constexpr uint64_t kMostSums = 1u << 24;

// Which kernel, and in how many pieces of k: the one that is expected to take the least time (us).  A tile kernel's
// workgroups run in rounds of as many as the 256 compute units hold; a round takes a fixed time and one per stage of
// 128 bytes of k, longer where several workgroups share a compute unit.  Few rows: the weights' bytes, a's rows that
// every workgroup reads anew, and the turns of a wavefront.  Fitted to 71 products from 1 x 1024 x 1024 to 8192^3 that
// every kernel was timed on: the choice takes at most 6% longer than the fastest on 66 of them, 20% on the worst
// (us, the choice and the fastest: 8 x 500 x 300 5.4 and 4.5, 1500 x 1500 x 4096 22.0 and 20.1, 1024 x 1024 x 32768 51.7 and
// 47.3, 64 x 1024 x 8192 12.1 and 11.3, 3000 x 1500 x 700 12.3 and 11.6).
ProductPlan plan_product(uint32_t M, uint32_t N, uint32_t K) {
  struct Kernel { uint32_t kind, rows, cols, slots; double fixed, alone, full; };
  static constexpr Kernel kernels[] = {
      {kProductTile64Deep, 64, 64, 2, 2.3, 0.17, 0.37},
      {kProductTile64, 64, 64, 5, 1.9, 0.24, 1.2},
      {kProductTile128x64, 128, 64, 2, 2.25, 0.39, 0.57},
      {kProductTile128, 128, 128, 2, 3.2, 0.57, 0.97},
      {kProductTile256, 256, 256, 1, 11.4, 1.3, 1.3},
  };
  constexpr double kLaunch = 2.3, kCus = 256.0;
  // At most 64 of k (at 128 the loads of 32 bytes from each row cost more than stages) and many results (us, without stages and the
  // best tiles: 8192 x 8192 x 64 41.3 / 50.2, fp32 50.3 / 59.4; 3968 x 2517 x 34 9.8 / 12.7; 1536 x 1536 x 64 5.4 / 5.7; 1024 x 1024 x 64
  // 5.2 / 4.5; 8192 x 8192 x 128 68.4 / 49.3), in rows that fill a workgroup's (70000 x 64 x 64 8.1 / 7.8).
  if (K <= kShallowDepth && N >= kShallowCols && (uint64_t)M * N >= 1u << 21 &&
      (uint64_t)((M + kShallowRows - 1) / kShallowRows) * ((N + kShallowCols - 1) / kShallowCols) < 1u << 23)
    return {kProductShallow, 1, kMostK, 0};
  const uint32_t fewest = std::max(1u, (K + kMostK - 1) / kMostK);
  auto join = [&](uint32_t splits) { return splits > 1 ? 3.8 + 8.0 * splits * M * N / 7.4e6 : 0.0; };
  ProductPlan best = {};
  double least = 1e300;
  auto offer = [&](uint32_t kind, uint32_t splits, double us) {
    if (us >= least) return;
    least = us;
    const uint32_t piece = splits == 1 ? kMostK : ((K + splits - 1) / splits + 255) / 256 * 256;
    best = {kind, splits == 1 ? 1 : (K + piece - 1) / piece, piece, 0};
  };
  for (const Kernel& k : kernels) {
    const double tiles = (double)((M + k.rows - 1) / k.rows) * ((N + k.cols - 1) / k.cols), slots = kCus * k.slots;
    if (tiles >= 1 << 23 && k.kind != kProductTile256) continue;   // (a launch has fewer than 2^32 threads)
    for (uint32_t splits = fewest; splits <= kMorePieces * fewest; splits *= 2) {
      if (splits > fewest && (K <= kLeastK || K / splits < kLeastPiece || tiles * splits > 2 * kCus || (double)splits * M * N > kMostSums)) break;
      const double stages = std::ceil(K / 128.0 / splits), groups = tiles * splits;
      auto round = [&](double n) {
        const double share = k.slots == 1 ? 0.0 : std::max(0.0, std::ceil(n / kCus) - 1) / (k.slots - 1);
        return k.fixed + stages * (k.alone + share * (k.full - k.alone));
      };
      const double rounds = std::floor(groups / slots), left = groups - rounds * slots;
      offer(k.kind, splits, kLaunch + rounds * round(slots) + (left > 0 ? round(left) : 0.0) + join(splits));
    }
  }
  if (M <= 32 && N <= 1u << 25)   // (a launch has fewer than 2^32 threads, here too)
    offer(kProductFew, fewest, kLaunch + 1.4 + (double)N * K / 1.2e7 + (double)M * K * ((N + 15) / 16) / 1.4e7 + 0.65 * std::ceil(K / 2048.0) + join(fewest));
  if (best.splits > 1) best.bytes = (uint64_t)best.splits * M * N * 4;
  return best;
}

uint64_t product_space(uint64_t M, uint64_t N, uint64_t K) {
  const uint64_t fewest = std::max<uint64_t>(1, (K + kMostK - 1) / kMostK), least = fewest > 1 ? fewest * M * N : 0;
  if (K <= kLeastK) return 0;
  uint64_t splits = kMorePieces * fewest;
  while (fewest == 1 && K / splits < kLeastPiece) splits /= 2;
  return 4 * std::max(least, std::min(splits * M * N, kMostSums));
}

hipError_t launch_products(const ProductPair& pair, uint32_t kind, hipStream_t st) {
  const ProductArgs& a = pair.of[0];
  auto tiles = [&](auto kernel, uint32_t rows, uint32_t cols) {
    ProductPair p = pair;
    auto count = [&](const ProductArgs& x) { return (x.M + rows - 1) / rows * ((x.N + cols - 1) / cols); };
    p.first = count(a);
    const dim3 grid(p.first + (pair.count > 1 ? count(pair.of[1]) : 0), a.splits);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, p);
  };
  if (kind == kProductFew) {
    const uint32_t steps = (std::min(a.K, a.split_k) + kFewDepth - 1) / kFewDepth;
    const uint32_t waves = std::max(1u, std::min(steps, kFewWaves)), lds = 4096 * waves;
    const dim3 block(64 * waves), grid((a.N + 15) / 16, a.splits);
    if (a.M <= 16) hipLaunchKernelGGL(k_product_few<1>, grid, block, lds, st, a);
    else hipLaunchKernelGGL(k_product_few<2>, grid, block, lds, st, a);
  }
  else if (kind == kProductTile64Deep) tiles(k_product<1, 1, 4>, 64, 64);
  else if (kind == kProductTile64) tiles(k_product<1, 1, 2>, 64, 64);
  else if (kind == kProductTile128x64) tiles(k_product<2, 1, 2>, 128, 64);
  else if (kind == kProductTile128) tiles(k_product<2, 2, 2>, 128, 128);
  else if (kind == kProductShallow) tiles(k_product_shallow, kShallowRows, kShallowCols);
  else tiles(k_product<4, 4, 2>, 256, 256);
  return hipGetLastError();
}

// Whether quantizing in every workgroup is the faster way: not where many of them make many levels each, or where the
// weights have so many rows that the kernels without it read them faster (us, together and apart, bf16, M x N x K: 1 x 4096 x 4096
// 8.4 / 11.3, 8 x 4096 x 4096 9.6 / 11.4, 1 x 12288 x 8192 22.9 / 24.1, 1 x 16384 x 4096 18.3 / 16.7, 1 x 28672 x 8192 49.4 / 45.5,
// 4 x 16384 x 2048 10.5 / 12.2, 2 x 32768 x 2048 15.6 / 16.3, 1 x 65536 x 512 12.9 / 11.4, 16 x 8192 x 2048 12.0 / 11.1).
// LDS holds 16 KiB of sums and 47 KiB of levels.
bool linear_few_fits(uint32_t M, uint32_t N, uint32_t K) {
  return M <= 16 && (N <= 12288 || (N <= 32768 && K <= 2048)) && K > 0 && (uint64_t)M * (K + 272) <= 47u << 10 &&
         (uint64_t)M * K * ((N + 15) / 16) <= 12u << 20;
}

hipError_t launch_linear_few(const LinearArgs& l, uint32_t type, bool stochastic, hipStream_t st) {
  const ProductArgs& a = l.product;
  const uint32_t steps = (a.K + kFewDepth - 1) / kFewDepth, waves = std::max(4u, std::min(steps, 16u));
  const uint32_t lds = 1024 * waves + a.M * (steps * kFewDepth + 16);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((a.N + 15) / 16), dim3(64 * waves), lds, st, l); };
  if (type == QSGD_TYPE_F32) stochastic ? go(k_linear_few<QSGD_TYPE_F32, true>) : go(k_linear_few<QSGD_TYPE_F32, false>);
  else if (type == QSGD_TYPE_BF16) stochastic ? go(k_linear_few<QSGD_TYPE_BF16, true>) : go(k_linear_few<QSGD_TYPE_BF16, false>);
  else stochastic ? go(k_linear_few<QSGD_TYPE_F16, true>) : go(k_linear_few<QSGD_TYPE_F16, false>);
  return hipGetLastError();
}

hipError_t launch_product_join(const ProductArgs& a, hipStream_t st) {
  const uint64_t units = (uint64_t)a.M * a.N / (a.N % 4 ? 1 : 4);
  const dim3 grid((uint32_t)std::min<uint64_t>((units + 255) / 256, kMostJoinBlocks));
  if (a.N % 4 == 0) hipLaunchKernelGGL(k_product_join<4>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_product_join<1>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace qsgd
