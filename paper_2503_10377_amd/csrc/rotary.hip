// Rotary positions: the pairs of a head turned by an angle that grows with the
// row's position, for the queries and keys of a chunk in one launch; turned
// the other way it is the gradient.
#include "row_common.h"

namespace sppo {
namespace {

constexpr int kWaves = 4;

// cos and sin of 2 pi a / 2^32: the nearest quarter turn goes, x in [-pi/4,
// pi/4] is left, where the Taylor series end below 2^-25 of their values
// (sin: x^11 / 11! = 1.8e-9; cos: x^12 / 12! = 1.2e-10).  The angle itself
// rounds twice (2^-24 of x each).
__device__ __forceinline__ void turn_cos_sin(uint32_t a, float& c, float& s) {
  const uint32_t q = (a + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(a - (q << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float y = x * x;
  const float sp = x + x * y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880))));
  const float cp = 1.f + y * (-.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 + y * (-1.f / 3628800)))));
  const float u = q & 1 ? sp : cp, v = q & 1 ? cp : sp;
  c = (q == 1 || q == 2) ? -u : u;
  s = q >= 2 ? -v : v;
}

// P consecutive elements as they lie in memory.
template <typename T, int P>
struct Piece;
template <>
struct Piece<uint16_t, 8> {
  u32x4 v;
  __device__ __forceinline__ void get(float (&f)[8]) const { unpack8(v, f); }
  __device__ __forceinline__ void set(const float (&f)[8]) { v = pack8(f); }
};
template <>
struct Piece<uint16_t, 4> {
  u32x2 v;
  __device__ __forceinline__ void get(float (&f)[4]) const {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      f[2 * e] = __uint_as_float(v[e] << 16);
      f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[4]) { v = pack_bf16x4(f[0], f[1], f[2], f[3]); }
};
template <int P>
struct Piece<float, P> {
  f32x4 v[P / 4];
  __device__ __forceinline__ void get(float (&f)[P]) const {
#pragma unroll
    for (int e = 0; e < P; ++e) f[e] = v[e >> 2][e & 3];
  }
  __device__ __forceinline__ void set(const float (&f)[P]) {
#pragma unroll
    for (int e = 0; e < P; ++e) v[e >> 2][e & 3] = f[e];
  }
};

// The U x 64 items from `base` on of one row: G groups of P pairs a head, then
// groups of 2 P copied elements; an item is two pieces of P elements.
template <typename T, int P, bool HALF, int U>
__device__ __forceinline__ void turn_items(const RotaryTensor& t, int rot, int64_t row, int base, int lane,
                                           const float* cs, const float* sn) {
  const int G = rot / 2 / P;
  const T* x = static_cast<const T*>(t.x) + row * t.ldx;
  T* y = static_cast<T*>(t.y) + row * t.ldy;
  Piece<T, P> a[U], b[U];
  int head[U], r[U], oa[U], ob[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int item = min(base + 64 * u + lane, t.items - 1);
    head[u] = (int)fast_div((uint32_t)item, t.per_head);
    r[u] = item - head[u] * t.per;
    oa[u] = r[u] * (HALF ? P : 2 * P);
    ob[u] = oa[u] + (HALF ? rot / 2 : P);
    if (HALF && r[u] >= G) {
      oa[u] = rot + (r[u] - G) * 2 * P;
      ob[u] = oa[u] + P;
    }
    const T* h = x + head[u] * t.hsx;
    a[u] = *reinterpret_cast<const Piece<T, P>*>(h + oa[u]);
    b[u] = *reinterpret_cast<const Piece<T, P>*>(h + ob[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (base + 64 * u + lane >= t.items) continue;
    if (r[u] < G) {
      float f[P], g[P], c[P], s[P];
      a[u].get(f);
      b[u].get(g);
#pragma unroll
      for (int e = 0; e < P; e += 4) {
        const f32x4 cv = *reinterpret_cast<const f32x4*>(cs + r[u] * P + e);
        const f32x4 sv = *reinterpret_cast<const f32x4*>(sn + r[u] * P + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[e + i] = cv[i], s[e + i] = sv[i];
      }
      if constexpr (HALF) {
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float p = f[e], q = g[e];
          f[e] = p * c[e] - q * s[e];
          g[e] = q * c[e] + p * s[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < P / 2; ++e) {
          const float p = f[2 * e], q = f[2 * e + 1], v = g[2 * e], w = g[2 * e + 1];
          f[2 * e] = p * c[e] - q * s[e];
          f[2 * e + 1] = q * c[e] + p * s[e];
          g[2 * e] = v * c[P / 2 + e] - w * s[P / 2 + e];
          g[2 * e + 1] = w * c[P / 2 + e] + v * s[P / 2 + e];
        }
      }
      a[u].set(f);
      b[u].set(g);
    }
    T* h = y + head[u] * t.hsy;
    *reinterpret_cast<Piece<T, P>*>(h + oa[u]) = a[u];
    *reinterpret_cast<Piece<T, P>*>(h + ob[u]) = b[u];
  }
}

// A wave makes the cosines and sines of its row in LDS, a pair a lane, and
// turns U x 64 items of one tensor with them.  The angle is position * freq
// modulo 2^64, of which the upper half is used.
template <int P, bool HALF, int U>
__global__ __launch_bounds__(64 * kWaves) void rotary_kernel(RotaryArgs a, uint32_t chunks, FastDiv by_chunks,
                                                             uint32_t waves) {
  extern __shared__ float tab[];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const uint32_t w = blockIdx.x * kWaves + wv;
  const uint32_t at = __builtin_amdgcn_readfirstlane(w < waves ? w : waves - 1);
  const uint32_t row = __builtin_amdgcn_readfirstlane(fast_div(at, by_chunks));
  const int c = (int)(at - row * chunks), pairs = a.rot / 2;
  uint64_t pos = (uint64_t)a.row0 + row;
  if (a.pos)
    pos = a.id64 ? (uint64_t) static_cast<const int64_t*>(a.pos)[row]
                 : (uint64_t)(int64_t) static_cast<const int32_t*>(a.pos)[row];
  float* cs = tab + wv * a.rot;
  float* sn = cs + pairs;
  for (int j = lane; j < pairs; j += 64) {
    float co, si;
    turn_cos_sin((uint32_t)((pos * a.freqs[j]) >> 32), co, si);
    cs[j] = a.amp * co;
    sn[j] = a.amp * a.sign * si;
  }
  __syncthreads();
  if (w >= waves) return;
  int k = 0;
  while (k + 1 < a.n && c >= a.t[k + 1].chunk0) ++k;
  const RotaryTensor& t = a.t[k];
  const int base = (c - t.chunk0) * 64 * U;
  if (t.f32)
    turn_items<float, P, HALF, U>(t, a.rot, row, base, lane, cs, sn);
  else
    turn_items<uint16_t, P, HALF, U>(t, a.rot, row, base, lane, cs, sn);
}

template <int P, int U>
hipError_t launch(RotaryArgs a, hipStream_t stream) {
  int64_t chunks = 0;
  for (int k = 0; k < a.n; ++k) {
    RotaryTensor& t = a.t[k];
    t.per = a.rot / 2 / P + (t.x == t.y ? 0 : (t.D - a.rot) / (2 * P));  // in place nothing is copied
    t.per_head = fast_divisor((uint32_t)t.per);
    t.items = t.heads * t.per;
    t.chunk0 = (int)chunks;
    chunks += (t.items + 64 * U - 1) / (64 * U);
  }
  // Waves of a launch index as numbers below 2^31 (fast_div).
  const int64_t rows_per = ((int64_t)1 << 30) / chunks;
  const FastDiv by_chunks = fast_divisor((uint32_t)chunks);
  const size_t lds = (size_t)kWaves * a.rot * sizeof(float);
  const int64_t rows = a.rows;
  for (int64_t r = 0; r < rows; r += rows_per) {
    RotaryArgs b = a;
    b.rows = rows - r < rows_per ? rows - r : rows_per;
    b.row0 = (int64_t)((uint64_t)a.row0 + (uint64_t)r);
    if (a.pos) b.pos = static_cast<const char*>(a.pos) + r * (a.id64 ? 8 : 4);
    for (int k = 0; k < a.n; ++k) {
      const int el = a.t[k].f32 ? 4 : 2;
      b.t[k].x = static_cast<const char*>(a.t[k].x) + r * a.t[k].ldx * el;
      b.t[k].y = static_cast<char*>(a.t[k].y) + r * a.t[k].ldy * el;
    }
    const uint32_t waves = (uint32_t)(b.rows * chunks);
    const dim3 grid((waves + kWaves - 1) / kWaves), block(64 * kWaves);
    if (a.half)
      hipLaunchKernelGGL((rotary_kernel<P, true, U>), grid, block, lds, stream, b, (uint32_t)chunks, by_chunks, waves);
    else
      hipLaunchKernelGGL((rotary_kernel<P, false, U>), grid, block, lds, stream, b, (uint32_t)chunks, by_chunks, waves);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, hipStream_t stream) {
  bool wide = a.rot % 16 == 0;
  for (int k = 0; k < a.n; ++k) wide = wide && a.t[k].D % 16 == 0;
  return wide ? launch<8, 4>(a, stream) : launch<4, 4>(a, stream);
}

}  // namespace sppo
