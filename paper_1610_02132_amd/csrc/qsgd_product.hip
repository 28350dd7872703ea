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

// A tile of 64 x 64 results to a workgroup, 32 x 32 to each of its wavefronts; 64 bytes of k at a time through LDS.
template <uint32_t TYPE>
__global__ __launch_bounds__(256) void k_product(ProductArgs a) {
  constexpr uint32_t kRow = 64 + 16;
  __shared__ __attribute__((aligned(16))) uint8_t as[64 * kRow], bs[64 * kRow];
  const uint32_t across = (a.N + 63) / 64, m0 = blockIdx.x / across * 64, n0 = blockIdx.x % across * 64;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t k0 = blockIdx.y * a.split_k, k1 = min(k0 + a.split_k, a.K);
  const uint32_t lr = threadIdx.x >> 2, lc = 16 * (threadIdx.x & 3);
  const uint32_t fm = 32 * (wave & 1) + (lane & 31), fn = 32 * (wave >> 1) + (lane & 31);
  int16v acc = {};
  for (uint32_t k = k0; k < k1; k += 64) {
    const uint4 va = operand(a.a, a.a_ld, m0 + lr, a.M, k + lc, a.K, true);
    const uint4 vb = operand(a.b, a.b_ld, n0 + lr, a.N, k + lc, a.K, false);
    __syncthreads();
    *reinterpret_cast<uint4*>(as + lr * kRow + lc) = va;
    *reinterpret_cast<uint4*>(bs + lr * kRow + lc) = vb;
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < 64; j += 32) {
      const int4v x = *reinterpret_cast<const int4v*>(as + fm * kRow + j + 16 * (lane >> 5));
      const int4v w = *reinterpret_cast<const int4v*>(bs + fn * kRow + j + 16 * (lane >> 5));
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, w, acc, 0, 0, 0);
    }
  }
  const uint32_t n = n0 + fn;
  if (n >= a.N) return;
#pragma unroll
  for (uint32_t i = 0; i < 16; ++i) {
    const uint32_t m = m0 + 32 * (wave & 1) + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
    if (m >= a.M) continue;
    if (a.part) a.part[((uint64_t)blockIdx.y * a.M + m) * a.N + n] = acc[i];
    else put<TYPE>(a, m, n, scaled((float)acc[i], a.a_scale[m], a.b_scale[n]));
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

hipError_t launch_product(const ProductArgs& a, hipStream_t st) {
  const dim3 grid((a.M + 63) / 64 * ((a.N + 63) / 64), a.splits);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (a.type == QSGD_TYPE_F32) go(k_product<QSGD_TYPE_F32>);
  else if (a.type == QSGD_TYPE_BF16) go(k_product<QSGD_TYPE_BF16>);
  else go(k_product<QSGD_TYPE_F16>);
  return hipGetLastError();
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
