// Rotary positions: the pairs of a head turned by an angle that grows with the
// row's position, for the queries and keys of a chunk in one launch; turned
// the other way it is the gradient.
//
// HBM-bound: 8192 rows of 32 + 32 heads of 128 bf16, on new data every time, in
// 47.5 us, 5.65 TB/s (16384 rows 89 us, 6.0); with 3001 rows of 32 bf16 and 8
// fp32 heads, half of each turned, 12.8 us.  A wave makes its row's angles once
// (a pair a lane) and turns one item a lane with them: with four items a lane the
// angles cost a quarter, but fewer waves' loads are on their way (52 us), and
// with the loads behind the table 48.
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

// P consecutive elements as they lie in memory: 16 bytes, or four bf16.
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
template <>
struct Piece<float, 4> {
  f32x4 v;
  __device__ __forceinline__ void get(float (&f)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = v[e];
  }
  __device__ __forceinline__ void set(const float (&f)[4]) { v = f32x4{f[0], f[1], f[2], f[3]}; }
};

// N cosines or sines from LDS.
template <int N>
__device__ __forceinline__ void angles(const float* p, float (&c)[N]) {
  typedef float V __attribute__((ext_vector_type(N < 4 ? N : 4)));
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    const V v = *reinterpret_cast<const V*>(p + e);
#pragma unroll
    for (int i = 0; i < (N < 4 ? N : 4); ++i) c[e + i] = v[i];
  }
}

// A piece with pairs side by side.
template <int P>
__device__ __forceinline__ void turn_pairs(float (&f)[P], const float* cs, const float* sn) {
  float c[P / 2], s[P / 2];
  angles(cs, c);
  angles(sn, s);
#pragma unroll
  for (int e = 0; e < P / 2; ++e) {
    const float a = f[2 * e], b = f[2 * e + 1];
    f[2 * e] = a * c[e] - b * s[e];
    f[2 * e + 1] = b * c[e] + a * s[e];
  }
}

// The cosines and sines of a row's pairs in a wave's part of LDS, a pair a lane.
// The angle is position * freq modulo 2^64, of which the upper half is used.
__device__ __forceinline__ void make_table(const RotaryArgs& a, uint64_t pos, int lane, float* cs, float* sn) {
  for (int j = lane; j < a.rot / 2; j += 64) {
    float c, s;
    turn_cos_sin((uint32_t)((pos * a.freqs[j]) >> 32), c, s);
    cs[j] = a.amp * c;
    sn[j] = a.amp * a.sign * s;
  }
  // Between the lanes of this wave only: its LDS accesses are served in order.
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// An item (64 of one row a wave) is two pieces of P elements of a head, half of
// what is turned (or half of what is copied) apart, so that neighbouring lanes'
// pieces lie side by side in either layout.  The loads go out before the table
// is made.
template <typename T, int P, bool HALF, bool PAST>
__device__ __forceinline__ void turn_item(const RotaryArgs& a, const RotaryTensor& t, int64_t row, uint64_t pos,
                                          int item, int lane, float* cs, float* sn) {
  const int G = a.rot / 2 / P;  // items of a head that are turned
  const int at = min(item, t.items - 1), head = (int)fast_div((uint32_t)at, t.per_head), r = at - head * t.per;
  const bool turned = r < G;
  const int oa = (turned ? 0 : a.rot - G * P) + r * P, ob = oa + (turned ? a.rot / 2 : (t.D - a.rot) / 2);
  const T* x = static_cast<const T*>(t.x) + row * t.ldx + head * t.hsx;
  T* y = static_cast<T*>(t.y) + row * t.ldy + head * t.hsy;
  Piece<T, P> p, q;
  const auto* px = reinterpret_cast<const decltype(p.v)*>(x + oa);
  const auto* qx = reinterpret_cast<const decltype(q.v)*>(x + ob);
  p.v = PAST ? __builtin_nontemporal_load(px) : *px;
  q.v = PAST ? __builtin_nontemporal_load(qx) : *qx;
  make_table(a, pos, lane, cs, sn);
  if (item >= t.items) return;
  if (turned) {
    float f[P], g[P];
    p.get(f);
    q.get(g);
    if constexpr (HALF) {
      float c[P], s[P];
      angles(cs + r * P, c);
      angles(sn + r * P, s);
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const float u = f[e], v = g[e];
        f[e] = u * c[e] - v * s[e];
        g[e] = v * c[e] + u * s[e];
      }
    } else {
      const int j = r * P / 2;
      turn_pairs(f, cs + j, sn + j);
      turn_pairs(g, cs + a.rot / 4 + j, sn + a.rot / 4 + j);
    }
    p.set(f);
    q.set(g);
  }
  *reinterpret_cast<decltype(p.v)*>(y + oa) = p.v;
  *reinterpret_cast<decltype(q.v)*>(y + ob) = q.v;
}

// A wave turns 64 items of one tensor's row.
template <int P, bool HALF, bool PAST>
__global__ __launch_bounds__(64 * kWaves) void rotary_kernel(RotaryArgs a, uint32_t chunks, FastDiv by_chunks,
                                                             uint32_t waves) {
  extern __shared__ float tab[];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const uint32_t w = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + wv);
  if (w >= waves) return;
  const uint32_t row = __builtin_amdgcn_readfirstlane(fast_div(w, by_chunks));
  const int c = (int)(w - row * chunks);
  uint64_t pos = (uint64_t)a.row0 + row;
  if (a.pos)
    pos = a.id64 ? (uint64_t) static_cast<const int64_t*>(a.pos)[row]
                 : (uint64_t)(int64_t) static_cast<const int32_t*>(a.pos)[row];
  float* cs = tab + wv * a.rot;
  int k = 0;
  while (k + 1 < a.n && c >= a.t[k + 1].chunk0) ++k;
  const RotaryTensor& t = a.t[k];
  const int item = (c - t.chunk0) * 64 + lane;
  if (t.f32)
    turn_item<float, 4, HALF, PAST>(a, t, row, pos, item, lane, cs, cs + a.rot / 2);
  else
    turn_item<uint16_t, P, HALF, PAST>(a, t, row, pos, item, lane, cs, cs + a.rot / 2);
}

template <int P, bool PAST>
hipError_t launch(RotaryArgs a, hipStream_t stream) {
  int64_t chunks = 0;
  for (int k = 0; k < a.n; ++k) {
    RotaryTensor& t = a.t[k];
    const int p = t.f32 ? 4 : P;
    t.per = a.rot / 2 / p + (t.x == t.y ? 0 : (t.D - a.rot) / (2 * p));  // in place nothing is copied
    t.per_head = fast_divisor((uint32_t)t.per);
    t.items = t.heads * t.per;
    t.chunk0 = (int)chunks;
    chunks += (t.items + 63) / 64;
  }
  const int64_t rows_per = kMaxWaves / chunks;
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
    const auto kernel = a.half ? rotary_kernel<P, true, PAST> : rotary_kernel<P, false, PAST>;
    hipLaunchKernelGGL(kernel, grid, block, lds, stream, b, (uint32_t)chunks, by_chunks, waves);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, hipStream_t stream) {
  // Pieces of 16 bytes where bf16 tensors divide into pairs of them, else of 8
  // (24 of 128 turned: 55 us where the whole head takes 47.5).  Large tensors are
  // read past the caches, but written through them, as the attention reads them
  // next.
  bool wide = true, past = false;
  for (int k = 0; k < a.n; ++k) {
    const RotaryTensor& t = a.t[k];
    wide = wide && (t.f32 || (a.rot % 16 == 0 && t.D % 16 == 0));
    past = past || stream_activation(a.rows, (int64_t)t.heads * t.D, t.f32);
  }
  if (past) return wide ? launch<8, true>(a, stream) : launch<4, true>(a, stream);
  return wide ? launch<8, false>(a, stream) : launch<4, false>(a, stream);
}

}  // namespace sppo
