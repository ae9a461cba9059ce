// Dropout whose mask is drawn from the element's position (row_common.h), on
// its own and with a residual added; applied to a gradient it is the backward.
#include "row_common.h"

namespace sppo {
namespace {

constexpr int kThreads = 256, kUnroll = 4;
constexpr int64_t kMaxGroups = (int64_t)1 << 30;  // of a launch: below fast_div's 2^31

// A thread takes kUnroll groups of eight elements (one draw each), 256 groups
// apart so that a wave's accesses are consecutive; all loads go out first.
// FLAT: rows lie without gaps, so a group's place needs no division.
// HBM-bound: 8192 x 4096 bf16 with a residual, on new data every time, in 34
// us, 6.0 TB/s (read through the caches: 39).
template <typename T, bool FLAT, bool RES, bool PAST>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a, FastDiv per_row, uint32_t groups) {
  const Dropper drop(a.drop);
  const uint32_t cpr = (uint32_t)a.cols / 8;
  const uint64_t g0 = (uint64_t)a.drop.row0 * cpr;
  Eight<T> x[kUnroll], res[kUnroll];
  uint32_t g[kUnroll];
  int64_t row[kUnroll], col[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    g[u] = blockIdx.x * (kThreads * kUnroll) + kThreads * u + threadIdx.x;
    if (g[u] >= groups) continue;
    if constexpr (FLAT) {
      row[u] = 0;
      col[u] = (int64_t)g[u] * 8;
    } else {
      const uint32_t r = fast_div(g[u], per_row);
      row[u] = r;
      col[u] = (int64_t)(g[u] - r * cpr) * 8;
    }
    x[u].template read<PAST>(static_cast<const T*>(a.x) + row[u] * a.ldx + col[u]);
    if constexpr (RES) res[u].template read<PAST>(static_cast<const T*>(a.res) + row[u] * a.ldres + col[u]);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (g[u] >= groups) continue;
    float f[8];
    x[u].get(f);
    drop.apply(g0 + g[u], f);
    if constexpr (RES) {
      float r[8];
      res[u].get(r);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] += r[e];
    }
    Eight<T>::store(static_cast<T*>(a.y) + row[u] * a.ldy + col[u], f);
  }
}

template <typename T, bool PAST>
hipError_t launch(const DropoutArgs& a, hipStream_t stream) {
  const int64_t cpr = a.cols / 8, rows_per = kMaxGroups / cpr;
  const bool flat = a.ldx == a.cols && a.ldy == a.cols && (!a.res || a.ldres == a.cols);
  const FastDiv div = fast_divisor((uint32_t)cpr);
  for (int64_t r = 0; r < a.rows; r += rows_per) {
    DropoutArgs b = a;
    b.rows = a.rows - r < rows_per ? a.rows - r : rows_per;
    b.x = static_cast<const T*>(a.x) + r * a.ldx;
    if (a.res) b.res = static_cast<const T*>(a.res) + r * a.ldres;
    b.y = static_cast<T*>(a.y) + r * a.ldy;
    b.drop.row0 += r;
    const uint32_t groups = (uint32_t)(b.rows * cpr);
    const dim3 grid((groups + kThreads * kUnroll - 1) / (kThreads * kUnroll)), block(kThreads);
    if (flat && a.res)
      hipLaunchKernelGGL((dropout_kernel<T, true, true, PAST>), grid, block, 0, stream, b, div, groups);
    else if (flat)
      hipLaunchKernelGGL((dropout_kernel<T, true, false, PAST>), grid, block, 0, stream, b, div, groups);
    else if (a.res)
      hipLaunchKernelGGL((dropout_kernel<T, false, true, PAST>), grid, block, 0, stream, b, div, groups);
    else
      hipLaunchKernelGGL((dropout_kernel<T, false, false, PAST>), grid, block, 0, stream, b, div, groups);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  if (a.rows <= 0 || a.cols <= 0 || a.cols % 8) return hipErrorInvalidValue;
  if (stream_activation(a.rows, a.cols, a.f32))
    return a.f32 ? launch<float, true>(a, stream) : launch<uint16_t, true>(a, stream);
  return a.f32 ? launch<float, false>(a, stream) : launch<uint16_t, false>(a, stream);
}

}  // namespace sppo
