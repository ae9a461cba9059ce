// The update of a list of parameters: the norm of all gradients, and the AdamW
// step with states in 32 or in 8 bits.  A workgroup takes a tile of kOptTile
// elements of one tensor; both are bound by HBM.
#include "row_common.h"

namespace sppo {
namespace {

constexpr int kThreads = 256, kGroups = kOptTile / (8 * kThreads);  // of eight elements a thread

__device__ __forceinline__ float load1(const void* p, int64_t i, bool bf16) {
  return bf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_bf16(void* p, int64_t i, float v) {
  static_cast<__bf16*>(p)[i] = (__bf16)v;
}

// --------------------------------------------------------------- sum of squares
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  return v;
}
// Over the workgroup, in every thread of the first wave.
__device__ __forceinline__ double block_sum64(double v, double* lds) {
  v = wave_sum64(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <typename T>
__device__ __forceinline__ double square_groups(const T* g, int n) {
  Eight<T> x[kGroups];
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int e = 8 * (kThreads * u + threadIdx.x);
    if (e + 8 <= n) x[u].stream(g + e);
    else x[u].zero();
  }
  double s = 0.0;
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    float f[8];
    x[u].get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (double)f[e] * f[e];
  }
  return s;
}

// Squares of fp32 numbers are exact in fp64 and their sum neither overflows nor
// loses small gradients; workgroup b adds tiles b, b + gridDim, ... in order.
__global__ __launch_bounds__(kThreads) void sumsq_kernel(OptTable t, double* part) {
  __shared__ double lds[4];
  double s = 0.0;
  for (int64_t i = blockIdx.x; i < t.tiles; i += gridDim.x) {
    const OptTile at = t.tile[i];
    const OptDesc& d = t.desc[at.tensor];
    const int64_t e0 = (int64_t)at.tile * kOptTile;
    const int n = (int)min((int64_t)kOptTile, d.n - e0);
    const bool bf = d.flags & kOptGradBf16;
    int done = 0;
    if (d.flags & kOptVector) {
      s += bf ? square_groups(static_cast<const uint16_t*>(d.grad) + e0, n)
              : square_groups(static_cast<const float*>(d.grad) + e0, n);
      done = n & ~7;
    }
    for (int e = done + threadIdx.x; e < n; e += kThreads) {
      const double g = load1(d.grad, e0 + e, bf);
      s += g * g;
    }
  }
  s = block_sum64(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double* part, int n, float max_norm, float* out,
                                                        int64_t* steps) {
  __shared__ double lds[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) s += part[i];
  s = block_sum64(s, lds);
  if (threadIdx.x != 0) return;
  const double norm = sqrt(s);
  const bool ok = (float)norm < __builtin_inff();
  out[0] = (float)norm;
  out[1] = !ok ? 0.f : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
  if (steps && ok) ++*steps;
}

// ------------------------------------------------------------------------ AdamW
struct Coef {
  float b1, c1, b2, c2, im, ir, eps, lr, wd, f;
};

// False: the norm of the gradients is infinite or NaN and nothing is changed.
__device__ __forceinline__ bool coefficients(const AdamArgs& a, const OptDesc& d, Coef& c, int64_t& t) {
  c.f = 1.f;
  if (a.norm) {
    if (!(a.norm[0] < __builtin_inff())) return false;
    c.f = a.norm[1];
  }
  c.b1 = (float)a.beta1; c.c1 = (float)(1.0 - a.beta1);
  c.b2 = (float)a.beta2; c.c2 = (float)(1.0 - a.beta2);
  c.im = a.im; c.ir = a.ir;
  t = a.step;
  if (a.step_dev) {
    t = max((int64_t)1, (int64_t)((uint64_t)t + (uint64_t)*a.step_dev));
    c.im = (float)(1.0 / (1.0 - beta_power(a.beta1, t)));
    c.ir = (float)(1.0 / sqrt(1.0 - beta_power(a.beta2, t)));
  }
  c.eps = a.eps;
  c.lr = a.lr * d.lr_scale;
  if (a.lr_dev) c.lr *= *a.lr_dev;
  c.wd = d.weight_decay;
  return true;
}

// m and v forward, each operation rounded by itself, so that what an 8-bit state
// is rounded from does not depend on the compiler's choice of fused products.
__device__ __forceinline__ void moments(const Coef& c, float g, float& m, float& v) {
#pragma clang fp contract(off)
  g = g * c.f;
  m = c.b1 * m + c.c1 * g;
  v = c.b2 * v + c.c2 * (g * g);
}
// The parameter from m and r = sqrt(v).
__device__ __forceinline__ float stepped(const Coef& c, float p, float m, float r) {
  const float q = m * c.im / (r * c.ir + c.eps);
  return p - c.lr * (q + c.wd * p);
}

template <typename G, bool PBF>
__device__ __forceinline__ void adam_groups(const Coef& c, const OptDesc& d, int64_t e0, int n) {
  const G* g = static_cast<const G*>(d.grad) + e0;
  float* w = (PBF ? d.master : static_cast<float*>(d.param)) + e0;
  float* m = static_cast<float*>(d.m) + e0;
  float* v = static_cast<float*>(d.v) + e0;
  Eight<G> xg[kGroups];
  Eight<float> xw[kGroups], xm[kGroups], xv[kGroups];
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int e = 8 * (kThreads * u + threadIdx.x);
    if (e + 8 > n) continue;
    xg[u].load(g + e);
    xw[u].load(w + e);
    xm[u].load(m + e);
    xv[u].load(v + e);
  }
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int e = 8 * (kThreads * u + threadIdx.x);
    if (e + 8 > n) continue;
    float fg[8], fw[8], fm[8], fv[8];
    xg[u].get(fg);
    xw[u].get(fw);
    xm[u].get(fm);
    xv[u].get(fv);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      moments(c, fg[i], fm[i], fv[i]);
      fw[i] = stepped(c, fw[i], fm[i], sqrtf(fv[i]));
    }
    Eight<float>::store(m + e, fm);
    Eight<float>::store(v + e, fv);
    Eight<float>::store(w + e, fw);
    if constexpr (PBF) Eight<uint16_t>::store(static_cast<uint16_t*>(d.param) + e0 + e, fw);
  }
}

__global__ __launch_bounds__(kThreads) void adam_f32_kernel(OptTable tab, AdamArgs a) {
  const OptTile at = tab.tile[blockIdx.x];
  const OptDesc& d = tab.desc[at.tensor];
  const int64_t e0 = (int64_t)at.tile * kOptTile;
  const int n = (int)min((int64_t)kOptTile, d.n - e0);
  Coef c;
  int64_t t;
  if (!coefficients(a, d, c, t)) return;
  const bool pbf = d.flags & kOptParamBf16, gbf = d.flags & kOptGradBf16;
  int done = 0;
  if (d.flags & kOptVector) {
    if (gbf && pbf) adam_groups<uint16_t, true>(c, d, e0, n);
    else if (gbf) adam_groups<uint16_t, false>(c, d, e0, n);
    else if (pbf) adam_groups<float, true>(c, d, e0, n);
    else adam_groups<float, false>(c, d, e0, n);
    done = n & ~7;
  }
  float* w = pbf ? d.master : static_cast<float*>(d.param);
  float* m = static_cast<float*>(d.m);
  float* v = static_cast<float*>(d.v);
  for (int i = done + threadIdx.x; i < n; i += kThreads) {
    const int64_t e = e0 + i;
    float fm = m[e], fv = v[e];
    moments(c, load1(d.grad, e, gbf), fm, fv);
    const float fw = stepped(c, w[e], fm, sqrtf(fv));
    m[e] = fm;
    v[e] = fv;
    w[e] = fw;
    if (pbf) store_bf16(d.param, e, fw);
  }
}

// ---------------------------------------------------------------- 8-bit states
// 2^k of k in [-126, 127]; a block's exponent byte 0 stands for zeros.
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

__device__ __forceinline__ void decode8(u32x2 codes, float scale, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], true);
    f[4 * i] = lo[0] * scale;
    f[4 * i + 1] = lo[1] * scale;
    f[4 * i + 2] = hi[0] * scale;
    f[4 * i + 3] = hi[1] * scale;
  }
}

// The exponent of a block of 32 (eight elements in each of four neighbouring
// lanes): the least k >= -126 with the largest finite magnitude at most 448 2^k
// (448 = 1.75 2^8: mantissas above .75 carry into the exponent).
__device__ __forceinline__ int block_exponent(const float (&f)[8]) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = fabsf(f[i]);
    a = fmaxf(a, x < __builtin_inff() ? x : 0.f);
  }
  a = fmaxf(a, dpp<0xB1>(a));
  a = fmaxf(a, dpp<0x4E>(a));
  return max((int)((__float_as_uint(a) + 0x1FFFFFu) >> 23) - 135, -126);
}

// y >= 0, at most 448, cut to a multiple of its e4m3 step after 16 random bits
// were added in what is cut off (20 bits of the mantissa; below 2^-6, where the
// step stays 2^-9, of y + 2^-6).  Anything else becomes NaN.
__device__ __forceinline__ float round8(float y, uint32_t bits) {
  const float low = y < 0.015625f ? 0.015625f : 0.f;
  const uint32_t t = (__float_as_uint(y + low) + (bits << 4)) & 0xFFF00000u;
  return y <= 448.f ? __uint_as_float(t) - low : __builtin_nanf("");
}

__device__ __forceinline__ u32x2 encode8(const float (&f)[8]) {
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
    r[i] = (uint32_t)w;
  }
  return r;
}

// The groups of a tile: elements from n on count as zeros and are not written,
// so every lane takes part in its block's exponent.
template <typename G, bool PBF>
__device__ __forceinline__ void adam8_groups(const Coef& c, const OptDesc& d, int64_t e0, int n, int64_t t,
                                             uint64_t seed) {
  const G* g = static_cast<const G*>(d.grad) + e0;
  float* w = (PBF ? d.master : static_cast<float*>(d.param)) + e0;
  uint8_t* m = static_cast<uint8_t*>(d.m) + e0;
  uint8_t* v = static_cast<uint8_t*>(d.v) + e0;
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int e = 8 * (kThreads * u + threadIdx.x);
    const bool whole = e + 8 <= n;
    float fg[8] = {}, fw[8] = {}, fm[8] = {}, fr[8] = {};
    const int64_t block = (e0 + e) / 32;
    u32x2 cm = {0, 0}, cv = {0, 0};
    float sm = 0.f, sv = 0.f;
    if (e < n) {
      sm = __uint_as_float((uint32_t)d.m_scale[block] << 23);
      sv = __uint_as_float((uint32_t)d.v_scale[block] << 23);
    }
    if (whole) {
      Eight<G> xg;
      Eight<float> xw;
      xg.load(g + e);
      xw.load(w + e);
      xg.get(fg);
      xw.get(fw);
      cm = *reinterpret_cast<const u32x2*>(m + e);
      cv = *reinterpret_cast<const u32x2*>(v + e);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e + i < n) {
          fg[i] = load1(g, e + i, sizeof(G) == 2);
          fw[i] = w[e + i];
          cm[i >> 2] |= (uint32_t)m[e + i] << (8 * (i & 3));
          cv[i >> 2] |= (uint32_t)v[e + i] << (8 * (i & 3));
        }
    }
    decode8(cm, sm, fm);
    decode8(cv, sv, fr);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v2 = fr[i] * fr[i];
      moments(c, fg[i], fm[i], v2);
      fr[i] = sqrtf(v2);
      fw[i] = stepped(c, fw[i], fm[i], fr[i]);
    }
    const int km = block_exponent(fm), kr = block_exponent(fr);
    const float im = pow2(-km), ir = pow2(-kr);
    const uint64_t group = 8 * ((uint64_t)d.block0 + (uint64_t)block) + (uint64_t)((e & 31) >> 2);
    const u32x4 d0 = philox(group, (uint64_t)t, seed), d1 = philox(group + 1, (uint64_t)t, seed);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t word = i < 4 ? d0[i & 3] : d1[i & 3];
      fm[i] = copysignf(round8(fabsf(fm[i]) * im, word & 0xFFFFu), fm[i]);
      const float r = round8(fr[i] * ir, word >> 16);
      fr[i] = fr[i] > 0.f && r == 0.f ? 0.001953125f : r;
    }
    const u32x2 em = encode8(fm), er = encode8(fr);
    if (whole) {
      Eight<float>::store(w + e, fw);
      if constexpr (PBF) Eight<uint16_t>::store(static_cast<uint16_t*>(d.param) + e0 + e, fw);
      *reinterpret_cast<u32x2*>(m + e) = em;
      *reinterpret_cast<u32x2*>(v + e) = er;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e + i < n) {
          w[e + i] = fw[i];
          if constexpr (PBF) store_bf16(d.param, e0 + e + i, fw[i]);
          m[e + i] = (uint8_t)(em[i >> 2] >> (8 * (i & 3)));
          v[e + i] = (uint8_t)(er[i >> 2] >> (8 * (i & 3)));
        }
    }
    if (e < n && (e & 31) == 0) {
      d.m_scale[block] = (uint8_t)(km + 127);
      d.v_scale[block] = (uint8_t)(kr + 127);
    }
  }
}

__global__ __launch_bounds__(kThreads) void adam_e4m3_kernel(OptTable tab, AdamArgs a) {
  const OptTile at = tab.tile[blockIdx.x];
  const OptDesc& d = tab.desc[at.tensor];
  const int64_t e0 = (int64_t)at.tile * kOptTile;
  const int n = (int)min((int64_t)kOptTile, d.n - e0);
  Coef c;
  int64_t t;
  if (!coefficients(a, d, c, t)) return;
  const bool pbf = d.flags & kOptParamBf16, gbf = d.flags & kOptGradBf16;
  if (gbf && pbf) adam8_groups<uint16_t, true>(c, d, e0, n, t, a.seed);
  else if (gbf) adam8_groups<uint16_t, false>(c, d, e0, n, t, a.seed);
  else if (pbf) adam8_groups<float, true>(c, d, e0, n, t, a.seed);
  else adam8_groups<float, false>(c, d, e0, n, t, a.seed);
}

}  // namespace

hipError_t launch_grad_norm(const OptTable& t, float max_norm, float* out, int64_t* steps, double* part,
                            hipStream_t stream) {
  const int n = (int)(t.tiles < kNormBlocks ? t.tiles : kNormBlocks);
  if (n > 0) {
    hipLaunchKernelGGL(sumsq_kernel, dim3(n), dim3(kThreads), 0, stream, t, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, stream, part, n, max_norm, out, steps);
  return hipGetLastError();
}

hipError_t launch_adamw(const OptTable& t, int state, const AdamArgs& a, hipStream_t stream) {
  if (t.tiles <= 0 || t.tiles > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)t.tiles), block(kThreads);
  if (state == 2) hipLaunchKernelGGL(adam_e4m3_kernel, grid, block, 0, stream, t, a);
  else hipLaunchKernelGGL(adam_f32_kernel, grid, block, 0, stream, t, a);
  return hipGetLastError();
}

}  // namespace sppo
