// Cross-entropy of rows of logits and its gradient.
//   lse = log sum exp x,  loss = lse - (1 - e) x_t - e/V sum x + z lse^2
//   dx = w ((1 + 2 z lse) exp(x - lse) - (1 - e) [c = t] - e/V)
#include "row_common.h"

namespace sppo {
namespace {

__device__ __forceinline__ float element(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float element(const uint16_t* p, int64_t i) {
  return __uint_as_float((uint32_t)p[i] << 16);
}
__device__ __forceinline__ void put_element(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void put_element(uint16_t* p, int64_t i, float v) {
  reinterpret_cast<__bf16*>(p)[i] = (__bf16)v;
}

__device__ __forceinline__ int64_t target_of(const CeArgs& a, int64_t row) {
  const int64_t t = a.id64 ? static_cast<const int64_t*>(a.targets)[row] : static_cast<const int32_t*>(a.targets)[row];
  return t >= 0 && t < a.V ? t : -1;
}

// exp of x <= 0 (or of -inf, inf, NaN): the difference first, then one product.
__device__ __forceinline__ float exp_of(float d) { return fast_exp2(d * kLog2e); }

// A running maximum with the sum of exp(x - max) under it (max -inf or inf: the
// sum of exp(x), which is zero or infinite then).
struct Running {
  float m, s;
  __device__ __forceinline__ static float base(float m) { return fabsf(m) < __builtin_inff() ? m : 0.f; }
  __device__ __forceinline__ void join(float m2, float s2) {
    const float top = fmaxf(m, m2), b = base(top);
    // An empty side has the sum zero whatever its factor would be.
    const float f1 = s == 0.f ? 0.f : s * exp_of(base(m) - b), f2 = s2 == 0.f ? 0.f : s2 * exp_of(base(m2) - b);
    m = top;
    s = f1 + f2;
  }
};

template <typename T>
__device__ __forceinline__ void load_group(const T* x, int64_t g, int64_t V, float fill, float (&f)[8]) {
  Eight<T> v;
  v.load(x + 8 * g);
  v.get(f);
  const int left = (int)min((int64_t)8, V - 8 * g);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e >= left) f[e] = fill;
}

template <typename T>
__device__ __forceinline__ void store_group(T* y, int64_t g, int64_t V, const float (&f)[8]) {
  if (8 * g + 8 <= V) {
    Eight<T>::store(y + 8 * g, f);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (8 * g + e < V) put_element(y, 8 * g + e, f[e]);
}

// lse - (1 - e) x_t - e/V sum x + z lse^2 with lse = base + part, from the
// differences, so that what they have in common cancels first.
__device__ __forceinline__ float loss_of(const CeArgs& a, float base, float part, float xt, float sum) {
  float loss = part;
  if (a.smooth != 1.f) loss += (1.f - a.smooth) * (base - xt);
  if (a.smooth != 0.f) loss += a.smooth * (base - sum / (float)a.V);
  if (a.z != 0.f) loss += a.z * (base + part) * (base + part);
  return loss;
}

// A row's gradient: coef exp(x - base) - sm, and `hit` less at the target.
struct RowGradient {
  float base, coef, sm, hit;
  // exp(x - lse) as exp(x - max) / sum; from lse itself where there is no finite
  // maximum, or no sum (s <= 0).
  __device__ __forceinline__ RowGradient(const CeArgs& a, const Running& r, float lse, float factor) {
    const float w = factor * (a.scale_dev ? a.scale * *a.scale_dev : a.scale);
    const bool known = r.s > 0.f && fabsf(r.m) < __builtin_inff();
    base = known ? r.m : lse;
    coef = w * (a.z != 0.f ? 1.f + 2.f * a.z * lse : 1.f) / (known ? r.s : 1.f);
    sm = w * (a.smooth / (float)a.V);
    hit = w * (1.f - a.smooth);
  }
  // Of the eight elements of group g; t is the target, -1 where there is none.
  __device__ __forceinline__ void apply(float (&f)[8], int64_t g, int64_t t) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = coef * exp_of(f[e] - base) - sm;
    if (t >> 3 == g) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] -= (t & 7) == e ? hit : 0.f;
    }
  }
};

constexpr int kThreads = 1024, kWavesCe = kThreads / 64;

// A row a workgroup: one pass for the maximum and the sum, a second one, from
// the caches, for the gradient.
template <typename T>
__global__ __launch_bounds__(kThreads) void ce_stream_kernel(CeArgs a) {
  __shared__ float lm[kWavesCe], ls[kWavesCe], lx[kWavesCe];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  T* dx = a.dx ? static_cast<T*>(a.dx) + row * a.lddx : nullptr;
  const int64_t V = a.V, groups = (V + 7) / 8, t = target_of(a, row);
  if (t < 0) {
    if (threadIdx.x == 0) {
      a.loss[row] = 0.f;
      if (a.lse) a.lse[row] = 0.f;
    }
    const float zero[8] = {};
    for (int64_t g = threadIdx.x; dx && g < groups; g += kThreads) store_group(dx, g, V, zero);
    return;
  }
  const float xt = element(x, t);
  Running r{-__builtin_inff(), 0.f};
  float sum = 0.f;
  for (int64_t g = threadIdx.x; g < groups; g += kThreads) {
    float f[8];
    load_group(x, g, V, -__builtin_inff(), f);
    float top = f[0], s = 0.f;
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, f[e]);
    const float b = Running::base(top);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += exp_of(f[e] - b);
    r.join(top, s);
    if (a.smooth != 0.f) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += 8 * g + e < V ? f[e] : 0.f;
    }
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) r.join(__shfl_xor(r.m, k), __shfl_xor(r.s, k));
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) {
    lm[threadIdx.x >> 6] = r.m;
    ls[threadIdx.x >> 6] = r.s;
    lx[threadIdx.x >> 6] = sum;
  }
  __syncthreads();
  r = Running{lm[0], ls[0]};
  sum = lx[0];
  for (int k = 1; k < kWavesCe; ++k) {
    r.join(lm[k], ls[k]);
    sum += lx[k];
  }
  const float base = Running::base(r.m), part = logf(r.s), lse = base + part;
  if (threadIdx.x == 0) {
    a.loss[row] = loss_of(a, base, part, xt, sum);
    if (a.lse) a.lse[row] = lse;
  }
  if (!dx) return;
  const RowGradient rg(a, r, lse, 1.f);
  for (int64_t g = threadIdx.x; g < groups; g += kThreads) {
    float f[8];
    load_group(x, g, V, -__builtin_inff(), f);
    rg.apply(f, g, t);
    store_group(dx, g, V, f);
  }
}

constexpr int kThreadsBwd = 256, kGroupsBwd = 4;

// The gradient from a kept lse: kGroupsBwd groups a thread.
template <typename T>
__global__ __launch_bounds__(kThreadsBwd) void ce_bwd_kernel(CeArgs a, uint32_t parts, FastDiv by_parts) {
  const uint32_t row = fast_div(blockIdx.x, by_parts), part = blockIdx.x - row * parts;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  T* dx = static_cast<T*>(a.dx) + row * a.lddx;
  const int64_t V = a.V, groups = (V + 7) / 8, t = target_of(a, row);
  const RowGradient rg(a, Running{0.f, 0.f}, a.lse_in[row], a.dloss ? a.dloss[row] : 1.f);
#pragma unroll
  for (int u = 0; u < kGroupsBwd; ++u) {
    const int64_t g = ((int64_t)part * kGroupsBwd + u) * kThreadsBwd + threadIdx.x;
    if (g >= groups) continue;
    float f[8] = {};
    if (t >= 0) {
      load_group(x, g, V, 0.f, f);
      rg.apply(f, g, t);
    }
    store_group(dx, g, V, f);
  }
}

}  // namespace

size_t cross_entropy_workspace(int64_t, int64_t, bool) { return 0; }

hipError_t launch_cross_entropy(const CeArgs& a, hipStream_t stream) {
  if (a.rows <= 0 || a.rows > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)a.rows), block(kThreads);
  if (a.f32) hipLaunchKernelGGL(ce_stream_kernel<float>, grid, block, 0, stream, a);
  else hipLaunchKernelGGL(ce_stream_kernel<uint16_t>, grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cross_entropy_bwd(const CeArgs& a, hipStream_t stream) {
  const int64_t per = 8 * kGroupsBwd * kThreadsBwd, parts = (a.V + per - 1) / per;
  const int64_t rows_per = ((int64_t)1 << 30) / parts;
  const FastDiv by_parts = fast_divisor((uint32_t)parts);
  const int el = a.f32 ? 4 : 2, id = a.id64 ? 8 : 4;
  for (int64_t r = 0; r < a.rows; r += rows_per) {
    CeArgs b = a;
    b.rows = a.rows - r < rows_per ? a.rows - r : rows_per;
    b.x = static_cast<const char*>(a.x) + r * a.ldx * el;
    b.dx = static_cast<char*>(a.dx) + r * a.lddx * el;
    b.targets = static_cast<const char*>(a.targets) + r * id;
    b.lse_in = a.lse_in + r;
    if (a.dloss) b.dloss = a.dloss + r;
    const dim3 grid((uint32_t)(b.rows * parts)), block(kThreadsBwd);
    if (a.f32) hipLaunchKernelGGL(ce_bwd_kernel<float>, grid, block, 0, stream, b, (uint32_t)parts, by_parts);
    else hipLaunchKernelGGL(ce_bwd_kernel<uint16_t>, grid, block, 0, stream, b, (uint32_t)parts, by_parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace sppo
