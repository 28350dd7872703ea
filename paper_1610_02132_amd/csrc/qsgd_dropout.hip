// Dropout whose mask is drawn where it is needed and never stored:
//   y = residual + [h >= D] x 65536 / (65536 - D),
// h the 16-bit draw of the element.  A Philox block serves eight neighbouring columns of a row, so
// a lane takes eight columns: one 16-byte access per matrix for 16-bit types.  HBM bound: 8192 x 4096 bf16 with a
// residual 33.1 us = 6.1 TB/s, the rate of a plain copy.  One block to a lane: the wavefronts that wait for their
// loads are hidden by others (1, 2, 4, 8 blocks: 36.6, 37.7, 40.0, 44.7 us with ordinary loads and stores).
#include "qsgd_layer.hpp"

namespace qsgd {
namespace {

template <uint32_t TYPE, bool RESIDUAL, bool STREAM>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const uint32_t c8s = (a.cols + 7) / 8, iteration = draw_iteration(a.draws);
  const uint32_t u = blockIdx.x * 256 + threadIdx.x;   // (a call has fewer than 2^32 blocks, which is checked before the launch)
  if (u >= a.rows * c8s) return;
  const uint32_t r = u / c8s, c8 = u - r * c8s, c = 8 * c8, n = a.cols - c;
  Eight<TYPE> x, z, y;
  x.template load<STREAM>(element_at<TYPE>(a.x, a.x_ld, r, c), n);
  if (RESIDUAL) z.template load<STREAM>(element_at<TYPE>(a.residual, a.residual_ld, r, c), n);
  const HalfWords h = draw_block(a.draws, iteration, r, c8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v = half_word(h, i) >= a.drop ? x.value(i) * a.scale : 0.0f;
    if (RESIDUAL) v = z.value(i) + v;
    y.set(i, Element<TYPE>::narrow(v));
  }
  y.template store<STREAM>(element_at<TYPE>(a.y, a.y_ld, r, c), n);
}

}  // namespace

namespace {
template <uint32_t TYPE>
void launch_as(const DropoutArgs& a, bool stream, hipStream_t st) {
  const uint64_t units = (uint64_t)a.rows * ((a.cols + 7) / 8);
  const dim3 grid((uint32_t)((units + 255) / 256));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (a.residual) stream ? go(k_dropout<TYPE, true, true>) : go(k_dropout<TYPE, true, false>);
  else stream ? go(k_dropout<TYPE, false, true>) : go(k_dropout<TYPE, false, false>);
}
}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, uint32_t type, hipStream_t st) {
  // Past the caches where a matrix alone is larger than the 32 MiB of L2 and its rows are whole lines (8192 x 4096 bf16 with
  // a residual: 36.8 us with ordinary accesses, 33.1 past the caches; 5003 x 2049 fp32, rows across lines, 14.6 and 18.6).
  const uint32_t size = type == QSGD_TYPE_F32 ? 4 : 2;
  auto lines = [&](const void* p, uint64_t ld) { return (reinterpret_cast<uintptr_t>(p) | ld * size) % 128 == 0; };
  const bool stream = (uint64_t)a.rows * a.cols * size > 32ull << 20 && lines(a.x, a.x_ld) && lines(a.y, a.y_ld) &&
                      lines(a.residual, a.residual ? a.residual_ld : 0);
  if (type == QSGD_TYPE_F32) launch_as<QSGD_TYPE_F32>(a, stream, st);
  else if (type == QSGD_TYPE_BF16) launch_as<QSGD_TYPE_BF16>(a, stream, st);
  else launch_as<QSGD_TYPE_F16>(a, stream, st);
  return hipGetLastError();
}

}  // namespace qsgd
