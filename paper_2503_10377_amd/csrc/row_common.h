// Device-side helpers of the row-wise kernels: sums over a wave, eight
// elements of a row in and out, the counter-based generator of the dropout,
// and the division of a flat index by a row's pieces.
#pragma once

#include "sppo_kernels.h"
#include "tile_common.h"

namespace sppo {

// Sum over the wave, in every lane: DPP within the 16-lane rows (xor 1, xor 2,
// then mirrors, whose partners hold the other half's sum), permlane swaps
// between them; no LDS round trips.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  return sum_groups(v);
}

// The same over the N = 16, 32 or 64 consecutive lanes that hold a row.
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
  static_assert(N == 16 || N == 32 || N == 64, "");
  if constexpr (N == 64) return wave_sum(v);
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  if constexpr (N == 32) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// Four floats of a buffer whose caller promises a float's alignment.
using f32x4_a4 = float __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void unpack8(const u32x4& x, float (&f)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(x[e] << 16);
    f[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  const bf16x8 b = pack_bf16x8(f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]);
  return __builtin_bit_cast(u32x4, b);
}

// A row (the same for the whole wave) as a buffer of `bytes` bytes: lanes past
// its end read zeros and store nothing, so loads of a ragged row, or of one
// that isn't there (0 bytes), need no branch.  The compiler counts loads
// between branches exactly, and waits for all that are on their way behind a
// load that a branch may have passed by.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* p, int bytes) {
  return uniform_rsrc(reinterpret_cast<uint64_t>(p), __builtin_amdgcn_readfirstlane(bytes));
}
template <bool PAST>
__device__ __forceinline__ u32x4 load_row16(__amdgpu_buffer_rsrc_t row, int offset) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(row, offset, 0, PAST ? 2 : 0));
}

__device__ __forceinline__ float load_row4(__amdgpu_buffer_rsrc_t row) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(row, 0, 0, 0));
}
template <bool PAST>
__device__ __forceinline__ void store_row16(__amdgpu_buffer_rsrc_t row, int offset, const u32x4& v) {
  using raw = unsigned int __attribute__((ext_vector_type(4)));
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(raw, v), row, offset, 0, PAST ? 2 : 0);
}
// One float, from the lanes where `on`.
__device__ __forceinline__ void store_row4(__amdgpu_buffer_rsrc_t row, bool on, float v) {
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), row, on ? 0 : 4, 0, 0);
}

// Eight consecutive elements as they lie in memory, for activations of either
// type: bf16 in one 16-byte piece, fp32 in two.  Of large activations (see
// kStreamBytes) stream() reads what nobody reads again soon, so that it takes
// no place in the caches from what is written for the next kernel, and
// stream_out() writes what only a later kernel reads.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
  u32x4 v;
  __device__ __forceinline__ void zero() { v = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const uint16_t* p) { v = ld_global16(p); }
  __device__ __forceinline__ void stream(const uint16_t* p) {
    v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  }
  template <bool PAST>
  __device__ __forceinline__ void read(const uint16_t* p) {
    if constexpr (PAST) stream(p);
    else load(p);
  }
  template <bool PAST>
  __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t row, int c) {
    v = load_row16<PAST>(row, 2 * c);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const { unpack8(v, f); }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&f)[8]) {
    *reinterpret_cast<u32x4*>(p) = pack8(f);
  }
  template <bool PAST>
  static __device__ __forceinline__ void put(__amdgpu_buffer_rsrc_t row, int c, const float (&f)[8]) {
    store_row16<PAST>(row, 2 * c, pack8(f));
  }
  static __device__ __forceinline__ void stream_out(uint16_t* p, const float (&f)[8]) {
    __builtin_nontemporal_store(pack8(f), reinterpret_cast<u32x4*>(p));
  }
};
template <>
struct Eight<float> {
  f32x4 v[2];
  __device__ __forceinline__ void zero() { v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void load(const float* p) {
    v[0] = *reinterpret_cast<const f32x4*>(p);
    v[1] = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ __forceinline__ void stream(const float* p) {
    v[0] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
    v[1] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
  }
  template <bool PAST>
  __device__ __forceinline__ void read(const float* p) {
    if constexpr (PAST) stream(p);
    else load(p);
  }
  template <bool PAST>
  __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t row, int c) {
    v[0] = __builtin_bit_cast(f32x4, load_row16<PAST>(row, 4 * c));
    v[1] = __builtin_bit_cast(f32x4, load_row16<PAST>(row, 4 * c + 16));
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = v[e >> 2][e & 3];
  }
  static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
  }
  template <bool PAST>
  static __device__ __forceinline__ void put(__amdgpu_buffer_rsrc_t row, int c, const float (&f)[8]) {
    store_row16<PAST>(row, 4 * c, __builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]}));
    store_row16<PAST>(row, 4 * c + 16, __builtin_bit_cast(u32x4, f32x4{f[4], f[5], f[6], f[7]}));
  }
  static __device__ __forceinline__ void stream_out(float* p, const float (&f)[8]) {
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4*>(p + 4));
  }
};
__device__ __forceinline__ void load8f(const float* p, float (&f)[8]) {
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const f32x4 v = *reinterpret_cast<const f32x4_a4*>(p + e);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[e + i] = v[i];
  }
}

// a ^ b ^ c in one instruction.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): ten rounds of two
// 32 x 32 -> 64 bit products on a 128-bit counter, with a 64-bit key.  The
// products (v_mad_u64_u32, a quarter of the rate) are what it costs.  The seed
// has to be the same for the whole wave.
__device__ __forceinline__ u32x4 philox(uint64_t counter, uint64_t offset, uint64_t seed) {
  uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32);
  uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  // The rounds' keys are added up here, by the scalar unit: kept across a
  // kernel's loop they would take 18 scalar registers, which it then lacks.
  asm volatile("" : "+s"(k0), "+s"(k1));
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = xor3((uint32_t)(p1 >> 32), c1, k0);
    c1 = (uint32_t)p1;
    c2 = xor3((uint32_t)(p0 >> 32), c3, k1);
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

// The dropout of a kernel's rows: eight elements (one draw) at a time.
struct Dropper {
  uint64_t seed, offset;
  uint32_t t16;  // threshold in the high half word; 0: everything is kept
  float scale;   // of the kept elements
  __device__ __forceinline__ explicit Dropper(const DropArgs& d)
      : seed(d.seed), offset(d.offset), t16(d.threshold << 16), scale(d.threshold ? d.scale : 1.f) {
    if (d.offset_dev) offset += *d.offset_dev;
  }
  // The draw of the elements 8 g .. 8 g + 7 of the whole sequence, and with it:
  // the dropped ones of f become zero, the others are left for the caller to
  // scale.
  __device__ __forceinline__ u32x4 draw(uint64_t g) const { return philox(g, offset, seed); }
  __device__ __forceinline__ void keep(const u32x4& w, float (&f)[8]) const {
    const uint16_t t = (uint16_t)(t16 >> 16);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      f[e] = (e & 1 ? w[e >> 1] >= t16 : (uint16_t)w[e >> 1] >= t) ? f[e] : 0.f;
  }
  __device__ __forceinline__ void mask(uint64_t g, float (&f)[8]) const {
    if (t16 != 0) keep(draw(g), f);
  }
  __device__ __forceinline__ void apply(uint64_t g, float (&f)[8]) const {
    mask(g, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= scale;
  }
};

// n / d and n % d for n < 2^31 by a product with the rounded reciprocal that
// the host made.
__device__ __forceinline__ uint32_t fast_div(uint32_t n, const FastDiv& d) {
  return d.shift < 0 ? n : (uint32_t)(((uint64_t)n * d.mul) >> 32) >> d.shift;
}

}  // namespace sppo
