// Product of 8-bit matrices with a scale per row of each:
//   y[m][n] = (sum_k a[m][k] b[n][k]) a_scale[m] b_scale[n] + bias[n],
// both operands with k contiguous.  The sum is an integer and exact whatever the order, so that pieces of k
// can be summed apart (a workspace of int32 sums, joined in 64 bits) without changing the result.
#include "qsgd_layer.hpp"

namespace qsgd {
namespace {

using int4v = __attribute__((ext_vector_type(4))) int;
using int16v = __attribute__((ext_vector_type(16))) int;

// Most of k in one piece: 131008 * 128 * 128 < 2^31.
constexpr uint32_t kMostK = 131008;
constexpr uint32_t kSums = 99;   // "type" of a piece's sums in the workspace

// The sum times both scales, the smaller one first: an intermediate result overflows or vanishes only
// where the result does.  (A scale that is NaN compares false and stays.)
__device__ __forceinline__ float scaled(float sum, float s, float t) {
  const float lo = s < t ? s : t, hi = s < t ? t : s;
  return sum * lo * hi;
}

template <uint32_t TYPE>
__device__ __forceinline__ void put(const ProductArgs& a, uint32_t m, uint32_t n, float v) {
  if (a.bias) v += a.bias[n];
  *reinterpret_cast<typename Element<TYPE>::bits*>(element_at<TYPE>(a.y, a.y_ld, m, n)) =
      (typename Element<TYPE>::bits)Element<TYPE>::narrow(v);
}

// 16 bytes of an operand's row from k on; the row is clamped into the matrix (its results are not
// written), k into the row, where bytes behind K are zeroed in one of the operands.
__device__ __forceinline__ uint4 operand(const int8_t* p, uint64_t ld, uint32_t row, uint32_t rows, uint32_t k,
                                         uint32_t K, bool mask) {
  const uint32_t last = (K + 15) / 16 * 16 - 16, at = min(k, last);
  uint4 v = *reinterpret_cast<const uint4*>(p + (min(row, rows - 1) * ld + at));
  if (mask && k + 16 > K) {
    const uint32_t n = k < K ? K - k : 0u;   // valid bytes
    uint32_t* w = &v.x;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      const uint32_t have = n > 4 * j ? min(n - 4 * j, 4u) : 0u;
      w[j] &= have == 4 ? ~0u : (1u << (8 * have)) - 1u;
    }
  }
  return v;
}

// ---- tiles ------------------------------------------------------------------------
// A workgroup of four wavefronts makes a tile of 64 MI x 64 NI results, each wavefront 32 MI x 32 NI of them in
// registers (MFMA 32x32x32: the weights' rows are the rows, so that a lane holds four neighbouring results of
// one row of y).  64 bytes of k are a stage; four stages are in LDS, loaded straight from memory three and a half
// stages ahead.  Slot s of a row of 64 bytes holds chunk s ^ (row / 2 % 4), which spreads the 16-byte reads
// of eight rows over all banks.
constexpr uint32_t kDepth = 64;   // bytes of k in a stage

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
    if (LOADS) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);     // loads
    __builtin_amdgcn_sched_group_barrier(0x8, kEach, 0);             // matrix instructions
  }
  __builtin_amdgcn_sched_barrier(0);
}

template <int MI, int NI, uint32_t TYPE>
__global__ __launch_bounds__(256, MI * NI > 4 ? 1 : 2) void k_product(ProductArgs a) {
  constexpr uint32_t TM = 64 * MI, TN = 64 * NI, kStage = (TM + TN) * kDepth;
  constexpr int kLoads = MI + NI;   // of a wavefront and stage, 16 rows each
  __shared__ __attribute__((aligned(16))) uint8_t s0[kStage], s1[kStage], s2[kStage], s3[kStage];
  uint32_t tm, tn;
  place_tile(blockIdx.x, (a.M + TM - 1) / TM, (a.N + TN - 1) / TN, tm, tn);
  const uint32_t m0 = tm * TM, n0 = tn * TN;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t k0 = blockIdx.y * a.split_k, k1 = min(k0 + a.split_k, a.K);
  const uint32_t steps = (k1 - k0) / kDepth;
  const uint32_t rows_a = min(TM, a.M - m0), rows_b = min(TN, a.N - n0);
  const auto from_a = __builtin_amdgcn_make_buffer_rsrc((void*)(a.a + m0 * a.a_ld), 0, (int)((rows_a - 1) * (uint32_t)a.a_ld + (a.K + 15) / 16 * 16), 0x27000);
  const auto from_b = __builtin_amdgcn_make_buffer_rsrc((void*)(a.b + n0 * a.b_ld), 0, (int)((rows_b - 1) * (uint32_t)a.b_ld + (a.K + 15) / 16 * 16), 0x27000);
  uint32_t at_a[MI], at_b[NI];   // rows are clamped into the matrix
  const uint32_t chunk = 16 * ((lane & 3) ^ (lane >> 3 & 3));
#pragma unroll
  for (int i = 0; i < MI; ++i) at_a[i] = min(16u * (MI * wave + i) + (lane >> 2), rows_a - 1) * (uint32_t)a.a_ld + chunk;
#pragma unroll
  for (int i = 0; i < NI; ++i) at_b[i] = min(16u * (NI * wave + i) + (lane >> 2), rows_b - 1) * (uint32_t)a.b_ld + chunk;
  auto load = [&](uint32_t step, uint8_t* to) {
    const uint32_t k = k0 + step * kDepth;
#pragma unroll
    for (int i = 0; i < MI; ++i) load_to_lds(from_a, to + 1024 * (MI * wave + i), at_a[i], k);
#pragma unroll
    for (int i = 0; i < NI; ++i) load_to_lds(from_b, to + TM * kDepth + 1024 * (NI * wave + i), at_b[i], k);
  };
  const uint32_t wm = (wave & 1) * 32 * MI, wn = (wave >> 1) * 32 * NI;   // the wavefront's part of the tile
  const uint32_t frag = (lane & 31) * kDepth + 16 * ((lane >> 5) ^ (lane >> 1 & 3));
  int4v xf[2][MI], wf[2][NI];
  auto read = [&](const uint8_t* from, int half) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      wf[half][i] = *reinterpret_cast<const int4v*>(from + (TM + wn + 32 * i) * kDepth + (frag ^ (32 * half)));
#pragma unroll
    for (int i = 0; i < MI; ++i)
      xf[half][i] = *reinterpret_cast<const int4v*>(from + (wm + 32 * i) * kDepth + (frag ^ (32 * half)));
  };
  int16v acc[MI][NI] = {};
  auto multiply = [&](int half) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[half][j], xf[half][i], acc[i][j], 0, 0, 0);
  };
  // Stage `now` has its first half in registers when its step begins.  Behind the barrier all wavefronts have read
  // the stage and hold the next one's loads: its place is loaded again.
  auto step = [&](uint8_t* now, const uint8_t* next, uint32_t s) {
    read(now, 1);
    multiply(0);
    weave<MI * NI, MI + NI, 0>();
    wait_loads<2 * kLoads>();
    meet();
    load(s + 4, now);
    read(next, 0);
    multiply(1);
    weave<MI * NI, MI + NI, MI + NI>();
  };
  auto last_step = [&](uint8_t* now, const uint8_t* next, uint32_t s) {   // ... of the last seven, where loads end
    read(now, 1);
    multiply(0);
    weave<MI * NI, MI + NI, 0>();
    if (s + 3 < steps) wait_loads<2 * kLoads>();
    else if (s + 2 < steps) wait_loads<kLoads>();
    else wait_loads<0>();
    meet();
    if (s + 4 < steps) load(s + 4, now);
    read(next, 0);
    multiply(1);
  };
  if (steps > 0) {
    load(0, s0);
    if (steps > 1) load(1, s1);
    if (steps > 2) load(2, s2);
    if (steps > 3) { load(3, s3); wait_loads<3 * kLoads>(); }
    else if (steps > 2) wait_loads<2 * kLoads>();
    else if (steps > 1) wait_loads<kLoads>();
    else wait_loads<0>();
    meet();
    read(s0, 0);
    uint32_t s = 0;
    for (; s + 8 <= steps; s += 4) {
      step(s0, s1, s);
      step(s1, s2, s + 1);
      step(s2, s3, s + 2);
      step(s3, s0, s + 3);
    }
    for (; s < steps; s += 4) {
      last_step(s0, s1, s);
      if (s + 1 >= steps) break;
      last_step(s1, s2, s + 1);
      if (s + 2 >= steps) break;
      last_step(s2, s3, s + 2);
      if (s + 3 >= steps) break;
      last_step(s3, s0, s + 3);
    }
  }
  if (k0 + steps * kDepth < k1) {   // what is left of k, less than a stage: straight from memory, masked
#pragma unroll
    for (uint32_t half = 0; half < 2; ++half) {
      const uint32_t k = k0 + steps * kDepth + 32 * half + 16 * (lane >> 5);
#pragma unroll
      for (int i = 0; i < MI; ++i)
        xf[0][i] = __builtin_bit_cast(int4v, operand(a.a, a.a_ld, m0 + wm + 32 * i + (lane & 31), a.M, k, a.K, true));
#pragma unroll
      for (int i = 0; i < NI; ++i)
        wf[0][i] = __builtin_bit_cast(int4v, operand(a.b, a.b_ld, n0 + wn + 32 * i + (lane & 31), a.N, k, a.K, false));
      multiply(0);
    }
  }
  // The results leave through LDS, 32 rows of the wavefront's part at a time, so that a store covers whole lines.
  meet();   // (all wavefronts have read their last stage)
  constexpr uint32_t kSize = TYPE == QSGD_TYPE_F32 || TYPE == kSums ? 4 : 2;
  constexpr uint32_t kRow = 32 * NI * kSize + 16, kPer = 16 / kSize, kChunks = 32 * NI / kPer;   // bytes, results of 16 bytes, of which a row has
  constexpr uint32_t kBlock = 32 * kRow;                // then the part's scales and biases
  static_assert(kBlock + 2 * 32 * NI * 4 <= kStage, "");
  uint8_t* stage = wave == 0 ? s0 : wave == 1 ? s1 : wave == 2 ? s2 : s3;
  float* w_scale = reinterpret_cast<float*>(stage + kBlock);
  float* bias = w_scale + 32 * NI;
  if constexpr (TYPE != kSums) {
    for (uint32_t j = lane; j < 32 * NI; j += 64) {
      const uint32_t n = min(n0 + wn + j, a.N - 1);
      w_scale[j] = a.b_scale[n];
      bias[j] = a.bias ? a.bias[n] : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const uint32_t row0 = m0 + wm + 32 * i;
    float x_scale = 0.0f;
    if constexpr (TYPE != kSums) x_scale = a.a_scale[min(row0 + (lane & 31), a.M - 1)];
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint32_t w[4];
        const float4 ws = *reinterpret_cast<const float4*>(w_scale + 32 * j + 8 * g + 4 * (lane >> 5));
        const float4 bs = *reinterpret_cast<const float4*>(bias + 32 * j + 8 * g + 4 * (lane >> 5));
        const float each[4] = {ws.x, ws.y, ws.z, ws.w}, plus[4] = {bs.x, bs.y, bs.z, bs.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int sum = acc[i][j][4 * g + e];
          if constexpr (TYPE == kSums) w[e] = (uint32_t)sum;
          else {
            float v = scaled((float)sum, x_scale, each[e]);
            if (a.bias) v += plus[e];
            w[e] = Element<TYPE>::narrow(v);
          }
        }
        __builtin_amdgcn_sched_barrier(0);   // (one group's values in registers at a time)
        uint8_t* to = stage + (lane & 31) * kRow + (32 * j + 8 * g + 4 * (lane >> 5)) * kSize;
        if constexpr (kSize == 4) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(to) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
      }
    wait_loads<63>();   // (the wavefront's writes have arrived)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (uint32_t it = 0; it < kChunks / 2; ++it) {
      const uint32_t c = 64 * it + lane;
      const uint32_t row = c / kChunks, n = n0 + wn + c % kChunks * kPer, m = row0 + row;
      const uint4 v = *reinterpret_cast<const uint4*>(stage + row * kRow + c % kChunks * 16);
      if (m >= a.M || n >= a.N) continue;
      uint8_t* out = TYPE == kSums ? reinterpret_cast<uint8_t*>(a.part) + (((uint64_t)blockIdx.y * a.M + m) * a.N + n) * 4
                                   : reinterpret_cast<uint8_t*>(a.y) + (m * a.y_ld + n) * kSize;
      if (a.wide && n + kPer <= a.N) {
        *reinterpret_cast<uint4*>(out) = v;
      } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) {
          if (n + e >= a.N) break;
          if constexpr (kSize == 4) reinterpret_cast<uint32_t*>(out)[e] = w[e];
          else reinterpret_cast<uint16_t*>(out)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
        }
      }
    }
    wait_loads<63>();
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The pieces' sums of one result, added in 64 bits.
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_product_join(ProductArgs a) {
  const uint64_t all = (uint64_t)a.M * a.N;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256) {
    int64_t sum = 0;
    for (uint32_t s = 0; s < a.splits; ++s) sum += a.part[s * all + i];
    const uint32_t m = (uint32_t)(i / a.N), n = (uint32_t)(i % a.N);
    put<TYPE>(a, m, n, scaled((float)sum, a.a_scale[m], a.b_scale[n]));
  }
}

}  // namespace

ProductPlan plan_product(uint32_t M, uint32_t N, uint32_t K) {
  ProductPlan p = {1, kMostK, 0};
  if (K > kMostK) {
    p.splits = (K + kMostK - 1) / kMostK;
    p.bytes = (uint64_t)p.splits * M * N * 4;
  }
  return p;
}

namespace {
template <int MI, int NI>
hipError_t launch_tiles(const ProductArgs& a, hipStream_t st) {
  const dim3 grid((a.M + 64 * MI - 1) / (64 * MI) * ((a.N + 64 * NI - 1) / (64 * NI)), a.splits);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (a.part) go(k_product<MI, NI, kSums>);
  else if (a.type == QSGD_TYPE_F32) go(k_product<MI, NI, QSGD_TYPE_F32>);
  else if (a.type == QSGD_TYPE_BF16) go(k_product<MI, NI, QSGD_TYPE_BF16>);
  else go(k_product<MI, NI, QSGD_TYPE_F16>);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_product(const ProductArgs& a, hipStream_t st) {
  const uint64_t big = (uint64_t)((a.M + 255) / 256) * ((a.N + 255) / 256);
  return big >= 128 ? launch_tiles<4, 4>(a, st) : launch_tiles<2, 2>(a, st);
}

hipError_t launch_product_join(const ProductArgs& a, hipStream_t st) {
  const uint64_t blocks = ((uint64_t)a.M * a.N + 255) / 256;
  const dim3 grid((uint32_t)(blocks < 65536 ? blocks : 65536));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (a.type == QSGD_TYPE_F32) go(k_product_join<QSGD_TYPE_F32>);
  else if (a.type == QSGD_TYPE_BF16) go(k_product_join<QSGD_TYPE_BF16>);
  else go(k_product_join<QSGD_TYPE_F16>);
  return hipGetLastError();
}

}  // namespace qsgd
