// The update of a list of parameters: the norm of all gradients, and the AdamW
// step with states in 32 or in 8 bits.  A workgroup takes a tile of kOptTile
// elements of one tensor, whichever it belongs to, so a list of any tensors is one
// launch.  HBM-bound: 201M fp32 gradients' norm 125 us (6.4 TB/s), their AdamW
// step with fp32 states, masters and bf16 parameters (30 bytes an element) 1054 to
// 1085 us by the machine (5.6-5.7 TB/s); 50M parameters with 8-bit states and bf16
// gradients (16.1 bytes) 138 to 141 us (5.8 TB/s) with the vector units busy for
// 79%: ten rounds of the generator are a third of their work.  Tiles of 2048
// elements leave registers for eight waves a SIMD: with 4096 the 8-bit step took
// 145 us and 300 ragged tensors 8.5 instead of 7.5 (the norm 122), with 8192 242
// and 10.4.
//
// Four neighbouring elements a thread in one access: eight (two accesses of fp32,
// each of half the cache lines) took 1122 us, and 137 for the norm.  Accesses are
// aligned to the element only, which the hardware serves, so tensors off the
// 16-byte grid take the same path (300 ragged ones 8.3 us, element by element
// 11.6).  Lists whose gradients are 32 MiB and more in fp32 go past the caches in
// both directions (through them 1110 us, one direction 1105 and 1125, and the norm
// 137); the 8-bit codes, 4 bytes a thread, do not (140 -> 145 us).
#include "row_common.h"

namespace sppo {
namespace {

constexpr int kThreads = 256, kQuads = kOptTile / (4 * kThreads);  // of four elements a thread

// N consecutive elements of a tensor that is aligned to its element, in one
// access; PAST: past the caches.
template <typename T, int N>
struct Vec;
template <>
struct Vec<float, 4> {
  using V = f32x4_a4;
  V v;
  __device__ __forceinline__ void get(float (&f)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = v[e];
  }
  __device__ __forceinline__ void set(const float (&f)[4]) { v = V{f[0], f[1], f[2], f[3]}; }
};
template <>
struct Vec<uint16_t, 4> {
  using V = uint32_t __attribute__((ext_vector_type(2), aligned(2)));
  V v;
  __device__ __forceinline__ void get(float (&f)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
  }
  __device__ __forceinline__ void set(const float (&f)[4]) {
    const u32x2 p = pack_bf16x4(f[0], f[1], f[2], f[3]);
    v = V{p[0], p[1]};
  }
};
template <>
struct Vec<uint16_t, 8> {
  using V = uint32_t __attribute__((ext_vector_type(4), aligned(2)));
  V v;
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
  }
};
template <bool PAST, typename T, int N>
__device__ __forceinline__ void load_vec(Vec<T, N>& x, const T* p) {
  const auto* q = reinterpret_cast<const typename Vec<T, N>::V*>(p);
  x.v = PAST ? __builtin_nontemporal_load(q) : *q;
}
template <bool PAST, typename T>
__device__ __forceinline__ void store_quad(T* p, const float (&f)[4]) {
  Vec<T, 4> x;
  x.set(f);
  auto* q = reinterpret_cast<typename Vec<T, 4>::V*>(p);
  if constexpr (PAST) __builtin_nontemporal_store(x.v, q);
  else *q = x.v;
}

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *reinterpret_cast<__bf16*>(p) = (__bf16)v; }

// --------------------------------------------------------------- sum of squares
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  return v;
}
// Over a workgroup of WAVES waves, in every thread.
template <int WAVES>
__device__ __forceinline__ double block_sum64(double v) {
  __shared__ double lds[WAVES];
  v = wave_sum64(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = lds[0];
#pragma unroll
  for (int k = 1; k < WAVES; ++k) s += lds[k];
  return s;
}

// A tile's n <= kOptTile gradients.  Squares of fp32 numbers are exact in fp64,
// and their sum neither overflows nor loses small gradients.
template <typename T>
struct TileSquares {
  static constexpr int N = 16 / (int)sizeof(T), K = kOptTile / (N * kThreads);
  Vec<T, N> x[K];
  T rest;
  template <bool PAST>
  __device__ __forceinline__ void load(const T* g, int n) {
#pragma unroll
    for (int u = 0; u < K; ++u) {
      const int e = N * (kThreads * u + threadIdx.x);
      if (e + N <= n) load_vec<PAST>(x[u], g + e);
    }
    const int e = n / N * N + threadIdx.x;
    if (e < n) rest = g[e];
  }
  __device__ __forceinline__ double sum(int n) const {
    double s[2] = {0.0, 0.0};
#pragma unroll
    for (int u = 0; u < K; ++u) {
      const int e = N * (kThreads * u + threadIdx.x);
      if (e + N > n) continue;
      float f[N];
      x[u].get(f);
#pragma unroll
      for (int i = 0; i < N; ++i) s[i & 1] += (double)f[i] * f[i];
    }
    if (n / N * N + (int)threadIdx.x < n) {
      const double f = load1(&rest);
      s[0] += f * f;
    }
    return s[0] + s[1];
  }
};

// Workgroup b adds tiles b, b + gridDim, ... in order; where the next one lies is
// looked up while this one's gradients are on their way.
template <bool PAST>
__global__ __launch_bounds__(kThreads) void sumsq_kernel(OptTable t, double* part) {
  struct Place {
    const void* g;
    int n;
    bool bf16;
  };
  const auto place = [&](int64_t i) {
    const OptTile at = t.tile[min(i, t.tiles - 1)];
    const OptDesc& d = t.desc[at.tensor];
    const int64_t e0 = (int64_t)at.tile * kOptTile;
    const bool bf = d.flags & kOptGradBf16;
    return Place{static_cast<const char*>(d.grad) + e0 * (bf ? 2 : 4), (int)min((int64_t)kOptTile, d.n - e0), bf};
  };
  double s = 0.0;
  Place p = place(blockIdx.x);
  for (int64_t i = blockIdx.x; i < t.tiles; i += gridDim.x) {
    Place next;
    if (p.bf16) {
      TileSquares<uint16_t> x;
      x.template load<PAST>(static_cast<const uint16_t*>(p.g), p.n);
      next = place(i + gridDim.x);
      s += x.sum(p.n);
    } else {
      TileSquares<float> x;
      x.template load<PAST>(static_cast<const float*>(p.g), p.n);
      next = place(i + gridDim.x);
      s += x.sum(p.n);
    }
    p = next;
  }
  s = block_sum64<kThreads / 64>(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The partial sums, all loads at once.
constexpr int kNormThreads = 1024;
__global__ __launch_bounds__(kNormThreads) void norm_kernel(const double* part, int n, float max_norm, float* out,
                                                            int64_t* steps) {
  static_assert(kNormBlocks == 2 * kNormThreads, "");
  const int i = threadIdx.x, k = i + kNormThreads;
  const double a = i < n ? part[i] : 0.0, b = k < n ? part[k] : 0.0;
  const double s = block_sum64<kNormThreads / 64>(a + b);
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
  const float q = m * c.im * __builtin_amdgcn_rcpf(r * c.ir + c.eps);
  return p - c.lr * (q + c.wd * p);
}

// A tile with fp32 states: all loads first.
template <typename G, bool PBF, bool PAST>
__device__ __forceinline__ void adam_tile(const Coef& c, const OptDesc& d, int64_t e0, int n) {
  const G* g = static_cast<const G*>(d.grad) + e0;
  float* w = (PBF ? d.master : static_cast<float*>(d.param)) + e0;
  float* m = static_cast<float*>(d.m) + e0;
  float* v = static_cast<float*>(d.v) + e0;
  uint16_t* p = static_cast<uint16_t*>(d.param) + e0;
  Vec<G, 4> xg[kQuads];
  Vec<float, 4> xw[kQuads], xm[kQuads], xv[kQuads];
#pragma unroll
  for (int u = 0; u < kQuads; ++u) {
    const int e = 4 * (kThreads * u + threadIdx.x);
    if (e + 4 > n) continue;
    load_vec<PAST>(xg[u], g + e);
    load_vec<PAST>(xw[u], w + e);
    load_vec<PAST>(xm[u], m + e);
    load_vec<PAST>(xv[u], v + e);
  }
#pragma unroll
  for (int u = 0; u < kQuads; ++u) {
    const int e = 4 * (kThreads * u + threadIdx.x);
    if (e + 4 > n) continue;
    float fg[4], fw[4], fm[4], fv[4];
    xg[u].get(fg);
    xw[u].get(fw);
    xm[u].get(fm);
    xv[u].get(fv);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      moments(c, fg[i], fm[i], fv[i]);
      fw[i] = stepped(c, fw[i], fm[i], sqrtf(fv[i]));
    }
    store_quad<PAST>(m + e, fm);
    store_quad<PAST>(v + e, fv);
    store_quad<PAST>(w + e, fw);
    if constexpr (PBF) store_quad<PAST>(p + e, fw);
  }
  const int e = (n & ~3) + (int)threadIdx.x;
  if (e < n) {
    float fm = m[e], fv = v[e];
    moments(c, load1(g + e), fm, fv);
    const float fw = stepped(c, w[e], fm, sqrtf(fv));
    m[e] = fm;
    v[e] = fv;
    w[e] = fw;
    if constexpr (PBF) store1(p + e, fw);
  }
}

// ---------------------------------------------------------------- 8-bit states
// 2^k of k in [-126, 127]; a block's exponent byte 0 stands for zeros.
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

__device__ __forceinline__ void decode8(uint32_t codes, float scale, float (&f)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  f[0] = lo[0] * scale;
  f[1] = lo[1] * scale;
  f[2] = hi[0] * scale;
  f[3] = hi[1] * scale;
}
// The exponent of a block of 32 (four elements in each of eight neighbouring
// lanes): the least k >= -126 with the largest finite magnitude at most 448 2^k
// (448 = 1.75 2^8: mantissas above .75 carry into the exponent).
__device__ __forceinline__ float block_max(const float (&f)[4]) {
  float a = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));  // of what is no NaN
  a = fmaxf(a, dpp<0xB1>(a));
  a = fmaxf(a, dpp<0x4E>(a));
  return fmaxf(a, dpp<0x141>(a));
}
__device__ __forceinline__ int block_exponent(const float (&f)[4]) {
  float a = block_max(f);
  if (__builtin_amdgcn_ballot_w64(a == __builtin_inff())) {  // some block of the wave: rare
    float g[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = fabsf(f[i]) < __builtin_inff() ? f[i] : 0.f;
    a = block_max(g);
  }
  return max((int)((__float_as_uint(a) + 0x1FFFFFu) >> 23) - 135, -126);
}

// Four values under their block's power of two (or NaN, infinite) to codes, up
// with the probability of what is cut off: the conversion aligns the random
// word's 32 bits with what is below a code's last bit, also below the normal
// numbers, and carries.  HIGH: the draw's high halves, else the low ones.
template <bool HIGH>
__device__ __forceinline__ uint32_t encode8(const float (&f)[4], const u32x4& draw) {
  const auto bits = [&](int i) { return (int)(HIGH ? draw[i] & 0xFFFF0000u : draw[i] << 16); };
  int w = __builtin_amdgcn_cvt_sr_fp8_f32(f[0], bits(0), 0, 0);
  w = __builtin_amdgcn_cvt_sr_fp8_f32(f[1], bits(1), w, 1);
  w = __builtin_amdgcn_cvt_sr_fp8_f32(f[2], bits(2), w, 2);
  return (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(f[3], bits(3), w, 3);
}

// sqrt(v), zero below the normal numbers: one step of Newton's on v rsq(v) (2 ulp)
// leaves half an ulp and 2^-22 of one.
__device__ __forceinline__ float root(float v) {
  const float y = __builtin_amdgcn_rsqf(v), r = v * y;
  const float s = __builtin_fmaf(__builtin_fmaf(-r, r, v), 0.5f * y, r);
  return v < 1.17549435e-38f ? 0.f : s;
}

// Roots and steps of a quad some of whose v may be infinite (or NaN, by a beta2 of
// zero), though r and g are not: gradients from 1.8e19 on.  Those elements are
// computed from 2^-72 g, m, r and eps where one of g and r is above 2^60: squares
// below 2^112 and, where they count, normal numbers.  A beta2 below 2^-100 counts as
// zero there.  The others are what the plain path makes of them, times one.  States
// are kept to 240 2^120, the largest code's value that fp32 holds there: above it a
// code of 256 2^120 would be infinite.  (Without such an element no state grows
// that far.)
__device__ __forceinline__ void far_steps(const Coef& c, const float (&fg)[4], float (&fm)[4], const float (&v2)[4],
                                          float (&fr)[4], float (&fw)[4]) {
  const auto kept = [](float x) {
    constexpr float top = 0x1.ep127f;
    return fabsf(x) > top && fabsf(x) < __builtin_inff() ? copysignf(top, x) : x;
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool far = !(v2[i] < __builtin_inff());
    const float r0 = far && c.b2 < 0x1p-100f && fr[i] < __builtin_inff() ? 0.f : fr[i];
    const bool scaled = far && (r0 > 0x1p60f || fabsf(fg[i] * c.f) > 0x1p60f);
    const float s = scaled ? 0x1p-72f : 1.f;
    float unused = 0.f, v = (r0 * s) * (r0 * s);
    moments(c, fg[i] * s, unused, v);
    Coef d = c;
    d.eps = c.eps * s;
    const float r = root(v);
    fw[i] = stepped(d, fw[i], fm[i] * s, r);
    fr[i] = kept(scaled ? r * 0x1p72f : r);
    fm[i] = kept(fm[i]);
  }
}

// A tile with 8-bit states: elements from n on count as zeros and are not
// written, so that every lane takes part in its block's exponent.
template <typename G, bool PBF, bool PAST>
__device__ __forceinline__ void adam8_tile(const Coef& c, const OptDesc& d, int64_t e0, int n, int64_t t,
                                           uint64_t seed) {
  const G* g = static_cast<const G*>(d.grad) + e0;
  float* w = (PBF ? d.master : static_cast<float*>(d.param)) + e0;
  uint8_t* m = static_cast<uint8_t*>(d.m) + e0;
  uint8_t* v = static_cast<uint8_t*>(d.v) + e0;
  uint16_t* p = static_cast<uint16_t*>(d.param) + e0;
  uint8_t* ms = d.m_scale + e0 / 32;
  uint8_t* vs = d.v_scale + e0 / 32;
  const uint64_t group0 = 8 * (uint64_t)d.block0 + (uint64_t)e0 / 4;
  Vec<G, 4> xg[kQuads];
  Vec<float, 4> xw[kQuads];
  uint32_t cm[kQuads], cv[kQuads], sm[kQuads], sv[kQuads];
#pragma unroll
  for (int u = 0; u < kQuads; ++u) {
    const int q = kThreads * u + threadIdx.x, e = 4 * q;
    sm[u] = sv[u] = cm[u] = cv[u] = 0;
    xg[u].v = {};
    xw[u].v = {};
    if (e < n) {
      sm[u] = ms[q / 8];
      sv[u] = vs[q / 8];
    }
    if (e + 4 <= n) {
      load_vec<PAST>(xg[u], g + e);
      load_vec<PAST>(xw[u], w + e);
      cm[u] = *reinterpret_cast<const uint32_t*>(m + e);
      cv[u] = *reinterpret_cast<const uint32_t*>(v + e);
    }
  }
#pragma unroll
  for (int u = 0; u < kQuads; ++u) {
    const int q = kThreads * u + threadIdx.x, e = 4 * q;
    float fg[4], fw[4], fm[4], fr[4];
    xg[u].get(fg);
    xw[u].get(fw);
    const bool whole = e + 4 <= n, some = e < n && !whole;
    if (some) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e + i < n) {
          fg[i] = load1(g + e + i);
          fw[i] = w[e + i];
          cm[u] |= (uint32_t)m[e + i] << (8 * i);
          cv[u] |= (uint32_t)v[e + i] << (8 * i);
        }
    }
    decode8(cm[u], __uint_as_float(sm[u] << 23), fm);
    decode8(cv[u], __uint_as_float(sv[u] << 23), fr);
    float v2[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v2[i] = fr[i] * fr[i];
      moments(c, fg[i], fm[i], v2[i]);
    }
    const float top = max_nc(max3_nc(v2[0], v2[1], v2[2]), v2[3]);  // NaN where one is
    if (__builtin_amdgcn_ballot_w64(!(top < __builtin_inff()))) {    // some square of the wave: rare
      far_steps(c, fg, fm, v2, fr, fw);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fr[i] = root(v2[i]);
        fw[i] = stepped(c, fw[i], fm[i], fr[i]);
      }
    }
    const int km = block_exponent(fm), kr = block_exponent(fr);
    const float im = pow2(-km), ir = pow2(-kr);
    const u32x4 draw = philox(group0 + q, (uint64_t)t, seed);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      fm[i] *= im;
      fr[i] = fr[i] == 0.f ? 0.f : max_nc(fr[i] * ir, 0.001953125f);  // 2^-9: not to zero
    }
    const uint32_t em = encode8<false>(fm, draw), er = encode8<true>(fr, draw);
    if (whole) {
      store_quad<PAST>(w + e, fw);
      if constexpr (PBF) store_quad<PAST>(p + e, fw);
      *reinterpret_cast<uint32_t*>(m + e) = em;
      *reinterpret_cast<uint32_t*>(v + e) = er;
    } else if (some) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e + i < n) {
          w[e + i] = fw[i];
          if constexpr (PBF) store1(p + e + i, fw[i]);
          m[e + i] = (uint8_t)(em >> (8 * i));
          v[e + i] = (uint8_t)(er >> (8 * i));
        }
    }
    if (e < n && (q & 7) == 0) {
      ms[q / 8] = (uint8_t)(km + 127);
      vs[q / 8] = (uint8_t)(kr + 127);
    }
  }
}

template <bool SMALL, bool PAST>
__global__ __launch_bounds__(kThreads) void adam_kernel(OptTable tab, AdamArgs a) {
  const OptTile at = tab.tile[blockIdx.x];
  const OptDesc& d = tab.desc[at.tensor];
  const int64_t e0 = (int64_t)at.tile * kOptTile;
  const int n = (int)min((int64_t)kOptTile, d.n - e0);
  Coef c;
  int64_t t;
  if (!coefficients(a, d, c, t)) return;
  const bool pbf = d.flags & kOptParamBf16, gbf = d.flags & kOptGradBf16;
  if constexpr (SMALL) {
    if (gbf && pbf) adam8_tile<uint16_t, true, PAST>(c, d, e0, n, t, a.seed);
    else if (gbf) adam8_tile<uint16_t, false, PAST>(c, d, e0, n, t, a.seed);
    else if (pbf) adam8_tile<float, true, PAST>(c, d, e0, n, t, a.seed);
    else adam8_tile<float, false, PAST>(c, d, e0, n, t, a.seed);
  } else {
    if (gbf && pbf) adam_tile<uint16_t, true, PAST>(c, d, e0, n);
    else if (gbf) adam_tile<uint16_t, false, PAST>(c, d, e0, n);
    else if (pbf) adam_tile<float, true, PAST>(c, d, e0, n);
    else adam_tile<float, false, PAST>(c, d, e0, n);
  }
}

}  // namespace

hipError_t launch_grad_norm(const OptTable& t, float max_norm, float* out, int64_t* steps, double* part,
                            hipStream_t stream) {
  const int n = (int)(t.tiles < kNormBlocks ? t.tiles : kNormBlocks);
  if (n > 0) {
    if (stream_activation(t.tiles, kOptTile, true))
      hipLaunchKernelGGL(sumsq_kernel<true>, dim3(n), dim3(kThreads), 0, stream, t, part);
    else
      hipLaunchKernelGGL(sumsq_kernel<false>, dim3(n), dim3(kThreads), 0, stream, t, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kNormThreads), 0, stream, part, n, max_norm, out, steps);
  return hipGetLastError();
}

hipError_t launch_adamw(const OptTable& t, int state, const AdamArgs& a, hipStream_t stream) {
  if (t.tiles <= 0 || t.tiles > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)t.tiles), block(kThreads);
  const bool past = stream_activation(t.tiles, kOptTile, true), small = state == 2;
  if (small && past) hipLaunchKernelGGL((adam_kernel<true, true>), grid, block, 0, stream, t, a);
  else if (small) hipLaunchKernelGGL((adam_kernel<true, false>), grid, block, 0, stream, t, a);
  else if (past) hipLaunchKernelGGL((adam_kernel<false, true>), grid, block, 0, stream, t, a);
  else hipLaunchKernelGGL((adam_kernel<false, false>), grid, block, 0, stream, t, a);
  return hipGetLastError();
}

}  // namespace sppo
