// Dropout whose mask is drawn where it is needed and never stored:
//   y = residual + [h >= D] x 65536 / (65536 - D),
// h the 16-bit draw of the element.  A Philox block serves eight neighbouring columns of a row, so
// a lane takes eight columns: one 16-byte access per matrix for 16-bit types.  HBM bound.
#include "qsgd_layer.hpp"

namespace qsgd {
namespace {

constexpr uint32_t kUnits = 4;   // blocks of eight columns that a lane takes

template <uint32_t TYPE, bool RESIDUAL>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const uint32_t c8s = (a.cols + 7) / 8, iteration = draw_iteration(a.draws);
  const uint64_t units = (uint64_t)a.rows * c8s;
  const uint64_t u0 = (uint64_t)blockIdx.x * (256 * kUnits) + threadIdx.x;
  Eight<TYPE> x[kUnits], z[kUnits];
#pragma unroll
  for (uint32_t k = 0; k < kUnits; ++k) {
    const uint64_t u = u0 + k * 256;
    if (u >= units) continue;
    const uint32_t r = (uint32_t)(u / c8s), c = 8 * (uint32_t)(u % c8s), n = a.cols - c;
    x[k].load(element_at<TYPE>(a.x, a.x_ld, r, c), n, a.wide);
    if (RESIDUAL) z[k].load(element_at<TYPE>(a.residual, a.residual_ld, r, c), n, a.wide);
  }
#pragma unroll
  for (uint32_t k = 0; k < kUnits; ++k) {
    const uint64_t u = u0 + k * 256;
    if (u >= units) continue;
    const uint32_t r = (uint32_t)(u / c8s), c8 = (uint32_t)(u % c8s), c = 8 * c8, n = a.cols - c;
    const HalfWords h = draw_block(a.draws, iteration, r, c8);
    Eight<TYPE> y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v = half_word(h, i) >= a.drop ? x[k].value(i) * a.scale : 0.0f;
      if (RESIDUAL) v = z[k].value(i) + v;
      y.set(i, Element<TYPE>::narrow(v));
    }
    y.store(element_at<TYPE>(a.y, a.y_ld, r, c), n, a.wide);
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, uint32_t type, hipStream_t st) {
  const uint64_t units = (uint64_t)a.rows * ((a.cols + 7) / 8);
  const dim3 grid((uint32_t)((units + 256 * kUnits - 1) / (256 * kUnits)));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  const bool z = a.residual != nullptr;
  if (type == QSGD_TYPE_F32) z ? go(k_dropout<QSGD_TYPE_F32, true>) : go(k_dropout<QSGD_TYPE_F32, false>);
  else if (type == QSGD_TYPE_BF16) z ? go(k_dropout<QSGD_TYPE_BF16, true>) : go(k_dropout<QSGD_TYPE_BF16, false>);
  else z ? go(k_dropout<QSGD_TYPE_F16, true>) : go(k_dropout<QSGD_TYPE_F16, false>);
  return hipGetLastError();
}

}  // namespace qsgd
