// Cross-entropy of rows of logits and its gradient.
//   lse = log sum exp x,  loss = lse - (1 - e) x_t - e/V sum x + z lse^2
//   dx = w ((1 + 2 z lse) exp(x - lse) - (1 - e) [c = t] - e/V)
// HBM-bound where rows are many: each logit is read once and its gradient
// written once, if a row stays where it was read to.  Three kernels:
//   ce_row   a row in the registers of a wave or a workgroup, up to 131072 bf16
//            or 65536 fp32 logits (16 pieces of 16 bytes in each of 1024
//            threads).  8192 x 32768 bf16 181 us, 5.9 TB/s (two passes over
//            memory: 279), with the vector units at 70%.
//   ce_part, ce_grad   longer rows, and few long ones, a part of 16 KB a
//            workgroup: three trips to memory instead of two, but 1 x 131072
//            bf16 takes 7.3 us instead of 16.7, 64 x 131072 13.1 instead of 20,
//            301 x 200019 60 instead of 87 (one workgroup a row, two passes).
//   ce_bwd   the gradient from a kept lse, elementwise: 301 x 200019 bf16 40.8
//            us, 5.7 TB/s.
// A piece is 16 bytes and neighbouring lanes' pieces are neighbours: two
// 16-byte halves of eight fp32 elements a lane, as elsewhere here, left every
// access half a cache line (4096 x 32768 fp32: 205 -> 181 us), and halves written
// past the caches cost more than they save.
#include <algorithm>

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

// 16 bytes of a row as they lie in memory: N elements.
template <typename T>
struct Piece {
  static constexpr int N = 16 / (int)sizeof(T);
  u32x4 v;
  template <bool PAST>
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t row, int piece) {
    v = load_row16<PAST>(row, 16 * piece);
  }
  __device__ __forceinline__ void get(float (&f)[N]) const {
    if constexpr (N == 8) {
      unpack8(v, f);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = __uint_as_float(v[e]);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[N]) {
    if constexpr (N == 8) {
      v = pack8(f);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = __float_as_uint(f[e]);
    }
  }
  // The elements from `left` on become -inf.
  __device__ __forceinline__ void cut(int left) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (N == 8) {
        if (2 * e >= left) v[e] = 0xff80ff80u;
        else if (2 * e + 1 >= left) v[e] = (v[e] & 0xffffu) | 0xff800000u;
      } else {
        if (e >= left) v[e] = 0xff800000u;
      }
    }
  }
};

// Elements 0 .. left - 1 of a row's last piece.
template <typename T>
__device__ __forceinline__ void store_some(T* y, int left, const float (&f)[Piece<T>::N]) {
#pragma unroll
  for (int e = 0; e < Piece<T>::N; ++e)
    if (e < left) put_element(y, e, f[e]);
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
  // Of the N elements of a piece of which element t, if it is one, is the target.
  template <int N>
  __device__ __forceinline__ void apply(float (&f)[N], int t) const {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = coef * exp_of(f[e] - base) - sm;
    if ((uint32_t)t < (uint32_t)N) {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] -= t == e ? hit : 0.f;
    }
  }
};

// Maximum over the wave, in every lane.
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  v = fmaxf(v, dpp<0x140>(v));
  return max_groups(v);
}

// The wave's Running of its lanes'.
__device__ __forceinline__ Running wave_join(const Running& r) {
  const float top = wave_max(r.m);
  return {top, wave_sum(r.s == 0.f ? 0.f : r.s * exp_of(Running::base(r.m) - Running::base(top)))};
}

// K pieces of a row (or of n elements of one) a thread, TEAM apart: the maximum
// and the sum under it, without another trip to memory for the gradient.
template <typename T, int TEAM, int K>
struct RowPart {
  static constexpr int N = Piece<T>::N;
  Piece<T> v[K];
  // The last piece is read as a whole (a row's stride is in whole pieces), what
  // is past n does not count.
  template <bool PAST>
  __device__ __forceinline__ void load(const T* x, int lane, int n) {
    const int pieces = (n + N - 1) / N;
    const __amdgpu_buffer_rsrc_t row = row_buffer(x, 16 * pieces);
#pragma unroll
    for (int k = 0; k < K; ++k) v[k].template load<PAST>(row, lane + TEAM * k);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (TEAM * (k + 1) < pieces) continue;  // whole for the team
      const int left = n - N * (lane + TEAM * k);
      if (left < N) v[k].cut(left);
    }
  }
  // The compiler is not to keep what it unpacked in a pass for the next one,
  // which would take twice the registers.
  __device__ __forceinline__ void repack() {
    if constexpr (N == 8) {
#pragma unroll
      for (int k = 0; k < K; ++k) asm volatile("" : "+v"(v[k].v));
    }
  }
  // Whether the team has any of its k-th pieces: the same for all, so that rows
  // that fill few of the registers cost no passes over nothing (1000 x 70000 bf16
  // 82 -> 65 us, 8192 x 5000 38 -> 32).
  static __device__ __forceinline__ bool any(int k, int n) { return k == 0 || TEAM * N * k < n; }
  __device__ __forceinline__ Running running(int n) {
    Running r{-__builtin_inff(), 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!any(k, n)) break;
      float f[N];
      v[k].get(f);
#pragma unroll
      for (int e = 0; e < N; e += 2) r.m = max3_nc(r.m, f[e], f[e + 1]);
    }
    repack();
    const float b = Running::base(r.m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!any(k, n)) break;
      float f[N];
      v[k].get(f);
#pragma unroll
      for (int e = 0; e < N; ++e) r.s += exp_of(f[e] - b);
    }
    repack();
    return r;
  }
  __device__ __forceinline__ float sum(int lane, int n) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!any(k, n)) break;
      float f[N];
      v[k].get(f);
#pragma unroll
      for (int e = 0; e < N; ++e) s += N * (lane + TEAM * k) + e < n ? f[e] : 0.f;
    }
    repack();
    return s;
  }
  // The gradient; t: the target's place among the n elements, outside: none.
  template <bool PAST>
  __device__ __forceinline__ void gradient(const RowGradient& g, T* dx, int lane, int n, int64_t t) {
    const __amdgpu_buffer_rsrc_t out = row_buffer(dx, 16 * (n / N));  // pieces past it are not stored
    const int at = t >= 0 && t < n ? (int)t : -N * TEAM * K;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!any(k, n)) break;
      const int first = N * (lane + TEAM * k);
      float f[N];
      v[k].get(f);
      g.apply(f, at - first);
      v[k].set(f);
      store_row16<PAST>(out, first * (int)sizeof(T), v[k].v);
      if (TEAM * N * (k + 1) > n && n - first > 0 && n - first < N) store_some(dx + first, n - first, f);
    }
  }
  static __device__ __forceinline__ void zero(T* dx, int lane, int n) {
    for (int first = N * lane; first < n; first += N * TEAM) {
      const float f[N] = {};
      if (n - first < N) store_some(dx + first, n - first, f);
      else *reinterpret_cast<u32x4*>(dx + first) = u32x4{0, 0, 0, 0};
    }
  }
};

// What the waves of a workgroup found, joined; in every thread.
template <int WAVES>
__device__ __forceinline__ void block_join(Running& r, float& sum) {
  __shared__ float lds[3][WAVES];
  if ((threadIdx.x & 63) == 0) {
    lds[0][threadIdx.x >> 6] = r.m;
    lds[1][threadIdx.x >> 6] = r.s;
    lds[2][threadIdx.x >> 6] = sum;
  }
  __syncthreads();
  r = Running{lds[0][0], lds[1][0]};
  sum = lds[2][0];
#pragma unroll
  for (int k = 1; k < WAVES; ++k) {
    r.join(lds[0][k], lds[1][k]);
    sum += lds[2][k];
  }
}

// loss and lse of a row, the latter returned.
__device__ __forceinline__ float finish_row(const CeArgs& a, int64_t row, const Running& r, float xt, float sum,
                                            bool write) {
  const float base = Running::base(r.m), part = logf(r.s), lse = base + part;
  if (write) {
    a.loss[row] = loss_of(a, base, part, xt, sum);
    if (a.lse) a.lse[row] = lse;
  }
  return lse;
}
__device__ __forceinline__ void finish_nothing(const CeArgs& a, int64_t row) {
  a.loss[row] = 0.f;
  if (a.lse) a.lse[row] = 0.f;
}

// A row a team of threads, which keeps it in registers: one read, one write.
// Maximum and sum are taken by every thread under its own maximum and joined
// once.  PAST: logits are read and the gradient is written past the caches, from
// 32 MiB on; the products that read the gradient next are bound by their
// arithmetic (4096 x 32768 bf16 109 -> 100 us).
template <typename T, int TEAM, int K, bool PAST>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void ce_row_kernel(CeArgs a) {
  constexpr int ROWS = TEAM < 256 ? 256 / TEAM : 1;
  const int lane = threadIdx.x % TEAM, V = (int)a.V;
  const int64_t row = (int64_t)blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM);
  if (row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  T* dx = a.dx ? static_cast<T*>(a.dx) + row * a.lddx : nullptr;
  const int64_t t = target_of(a, row);
  if (t < 0) {
    if (lane == 0) finish_nothing(a, row);
    if (dx) RowPart<T, TEAM, K>::zero(dx, lane, V);
    return;
  }
  RowPart<T, TEAM, K> p;
  p.template load<PAST>(x, lane, V);
  const float xt = element(x, t);
  Running r = wave_join(p.running(V));
  float sum = a.smooth != 0.f ? wave_sum(p.sum(lane, V)) : 0.f;
  if constexpr (TEAM > 64) block_join<TEAM / 64>(r, sum);
  const float lse = finish_row(a, row, r, xt, sum, lane == 0);
  if (dx) p.template gradient<PAST>(RowGradient(a, r, lse, 1.f), dx, lane, V, t);
}

// Long rows in parts of kPart bytes, a workgroup each: every part leaves its
// maximum, the sum under it, its elements' sum and the target's element (which
// the gradient may overwrite), and the gradient's kernel joins a row's.
constexpr int kPartThreads = 256, kPartPieces = 4, kPart = 16 * kPartPieces * kPartThreads;

template <typename T>
__global__ __launch_bounds__(kPartThreads) void ce_part_kernel(CeArgs a, uint32_t parts, FastDiv by_parts) {
  const uint32_t row = fast_div(blockIdx.x, by_parts), part = blockIdx.x - row * parts;
  constexpr int E = kPart / (int)sizeof(T);
  const int64_t t = target_of(a, row), c0 = (int64_t)part * E;
  if (t < 0) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx + c0;
  const int n = (int)min((int64_t)E, a.V - c0);
  RowPart<T, kPartThreads, kPartPieces> p;
  p.template load<false>(x, threadIdx.x, n);
  const float xt = t >= c0 && t < c0 + n ? element(x, t - c0) : 0.f;
  Running r = wave_join(p.running(n));
  float sum = a.smooth != 0.f ? wave_sum(p.sum(threadIdx.x, n)) : 0.f;
  block_join<kPartThreads / 64>(r, sum);
  if (threadIdx.x == 0) static_cast<f32x4*>(a.workspace)[blockIdx.x] = f32x4{r.m, r.s, sum, xt};
}

// The gradient from the parts, of which the first workgroup of a row makes loss
// and lse too (the only one there is without a gradient).
template <typename T, bool PAST>
__global__ __launch_bounds__(kPartThreads) void ce_grad_kernel(CeArgs a, uint32_t parts, uint32_t grid_parts,
                                                               FastDiv by_parts) {
  const uint32_t row = fast_div(blockIdx.x, by_parts), part = blockIdx.x - row * grid_parts;
  constexpr int E = kPart / (int)sizeof(T);
  const int64_t t = target_of(a, row), c0 = (int64_t)part * E;
  const int n = (int)min((int64_t)E, a.V - c0);
  T* dx = a.dx ? static_cast<T*>(a.dx) + row * a.lddx + c0 : nullptr;
  using Part = RowPart<T, kPartThreads, kPartPieces>;
  if (t < 0) {
    if (part == 0 && threadIdx.x == 0) finish_nothing(a, row);
    if (dx) Part::zero(dx, threadIdx.x, n);
    return;
  }
  Part p;
  if (dx) p.template load<PAST>(static_cast<const T*>(a.x) + row * a.ldx + c0, threadIdx.x, n);
  const f32x4* q = static_cast<const f32x4*>(a.workspace) + (int64_t)row * parts;
  Running r{-__builtin_inff(), 0.f};
  float sum = 0.f;
  for (uint32_t i = threadIdx.x; i < parts; i += kPartThreads) {
    r.join(q[i][0], q[i][1]);
    sum += q[i][2];
  }
  r = wave_join(r);
  sum = wave_sum(sum);
  block_join<kPartThreads / 64>(r, sum);
  const float lse = finish_row(a, row, r, q[t / E][3], sum, part == 0 && threadIdx.x == 0);
  if (dx) p.template gradient<PAST>(RowGradient(a, r, lse, 1.f), dx, threadIdx.x, n, t - c0);
}

// The gradient from a kept lse: K x 64 pieces of a row a wave.
template <typename T, int K, bool PAST>
__global__ __launch_bounds__(256) void ce_bwd_kernel(CeArgs a, uint32_t parts, FastDiv by_parts) {
  const uint32_t wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const uint32_t row = fast_div(wave, by_parts), part = wave - row * parts;
  if (row >= a.rows) return;
  constexpr int E = 64 * K * Piece<T>::N;
  const int64_t t = target_of(a, row), c0 = (int64_t)part * E;
  const int n = (int)min((int64_t)E, a.V - c0);
  T* dx = static_cast<T*>(a.dx) + row * a.lddx + c0;
  if (t < 0) return RowPart<T, 64, K>::zero(dx, lane, n);
  RowPart<T, 64, K> p;
  p.template load<PAST>(static_cast<const T*>(a.x) + row * a.ldx + c0, lane, n);
  const RowGradient g(a, Running{0.f, 0.f}, a.lse_in[row], a.dloss ? a.dloss[row] : 1.f);
  p.template gradient<PAST>(g, dx, lane, n, t - c0);
}

// Rows [r, r + n) of a call.
CeArgs rows_from(const CeArgs& a, int64_t r, int64_t n) {
  const int el = a.f32 ? 4 : 2, id = a.id64 ? 8 : 4;
  CeArgs b = a;
  b.rows = n;
  b.x = static_cast<const char*>(a.x) + r * a.ldx * el;
  if (a.dx) b.dx = static_cast<char*>(a.dx) + r * a.lddx * el;
  b.targets = static_cast<const char*>(a.targets) + r * id;
  if (a.loss) b.loss = a.loss + r;
  if (a.lse) b.lse = a.lse + r;
  if (a.lse_in) b.lse_in = a.lse_in + r;
  if (a.dloss) b.dloss = a.dloss + r;
  return b;
}

int64_t parts_of(int64_t V, bool f32) { return (V * (f32 ? 4 : 2) + kPart - 1) / kPart; }

// Rows whose logits the gradient's kernel still finds in the memory-side cache
// (256 MB) after the parts' kernel: 1000 x 140000 bf16 takes 137 us with 160 MB
// at once, 140 with 96, 170 with 24 (the launches show); 300 x 1000000 fp32 532 us
// and 595 with all at once.
int64_t rows_at_once(int64_t rows, int64_t V, bool f32) {
  const int64_t fit = ((int64_t)160 << 20) / (V * (f32 ? 4 : 2));
  return std::min(rows, std::max<int64_t>(fit, 1));
}

// Below 128 rows a workgroup each leaves half of the compute units idle: 64 rows
// of 131072 bf16 take 20 us a row a workgroup and 13 in parts, 256 rows 29 and 36;
// rows of up to 32768 are too short for a second launch (64 rows 7.0 us).
constexpr int64_t kFewRows = 127;
bool in_parts(int64_t rows, int64_t V, bool f32) {
  if (V > (f32 ? 65536 : 131072)) return true;
  return V > 32768 && rows <= kFewRows;
}

template <typename T, bool PAST>
hipError_t launch_parts(const CeArgs& a, hipStream_t stream) {
  const int64_t parts = parts_of(a.V, a.f32), step = rows_at_once(a.rows, a.V, a.f32), n = a.dx ? parts : 1;
  const FastDiv by_parts = fast_divisor((uint32_t)parts), by_n = fast_divisor((uint32_t)n);
  for (int64_t r = 0; r < a.rows; r += step) {
    const CeArgs b = rows_from(a, r, std::min(step, a.rows - r));
    hipLaunchKernelGGL(ce_part_kernel<T>, dim3((uint32_t)(b.rows * parts)), dim3(kPartThreads), 0, stream, b,
                       (uint32_t)parts, by_parts);
    hipLaunchKernelGGL((ce_grad_kernel<T, PAST>), dim3((uint32_t)(b.rows * n)), dim3(kPartThreads), 0, stream, b,
                       (uint32_t)parts, (uint32_t)n, by_n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int TEAM, int K, bool PAST>
hipError_t launch_row(const CeArgs& a, hipStream_t stream) {
  constexpr int ROWS = TEAM < 256 ? 256 / TEAM : 1;
  constexpr int64_t step = kMaxWaves / (TEAM / 64);
  for (int64_t r = 0; r < a.rows; r += step) {
    const CeArgs b = rows_from(a, r, std::min(step, a.rows - r));
    hipLaunchKernelGGL((ce_row_kernel<T, TEAM, K, PAST>), dim3((uint32_t)((b.rows + ROWS - 1) / ROWS)),
                       dim3(TEAM * ROWS), 0, stream, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// As few pieces a thread as hold the row, at most 16, in the fewest threads that
// do: with 8 a compute unit holds four workgroups of 512 threads, whose loads,
// exponentials and stores overlap (4096 x 32768 bf16: 512 threads with 8 pieces
// 98 us, 256 with 16 102, 1024 with 4 103).  A workgroup that takes rows in turn,
// each written piece making room for the next row's, gains 3 to 10% on some sizes
// of 1024 threads and loses as much on others.
template <typename T, bool PAST>
hipError_t launch_loss(const CeArgs& a, hipStream_t stream) {
  if (in_parts(a.rows, a.V, a.f32)) return launch_parts<T, PAST>(a, stream);
  const int64_t pieces = (a.V + Piece<T>::N - 1) / Piece<T>::N;
  if (pieces <= 64) return launch_row<T, 64, 1, PAST>(a, stream);
  if (pieces <= 64 * 2) return launch_row<T, 64, 2, PAST>(a, stream);
  if (pieces <= 64 * 4) return launch_row<T, 64, 4, PAST>(a, stream);
  if (pieces <= 256 * 2) return launch_row<T, 256, 2, PAST>(a, stream);
  if (pieces <= 256 * 4) return launch_row<T, 256, 4, PAST>(a, stream);
  if (pieces <= 256 * 8) return launch_row<T, 256, 8, PAST>(a, stream);
  if (pieces <= 512 * 8) return launch_row<T, 512, 8, PAST>(a, stream);
  if (pieces <= 512 * 16) return launch_row<T, 512, 16, PAST>(a, stream);
  return launch_row<T, 1024, 16, PAST>(a, stream);
}

template <typename T, int K, bool PAST>
hipError_t launch_bwd(const CeArgs& a, hipStream_t stream) {
  constexpr int E = 64 * K * Piece<T>::N;
  const int64_t parts = (a.V + E - 1) / E, step = kMaxWaves / parts;
  const FastDiv by_parts = fast_divisor((uint32_t)parts);
  for (int64_t r = 0; r < a.rows; r += step) {
    const CeArgs b = rows_from(a, r, std::min(step, a.rows - r));
    const dim3 grid((uint32_t)((b.rows * parts + 3) / 4)), block(256);
    hipLaunchKernelGGL((ce_bwd_kernel<T, K, PAST>), grid, block, 0, stream, b, (uint32_t)parts, by_parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// One piece a lane where that is the row, so that no lane of a short row's wave
// computes on nothing.
template <typename T, bool PAST>
hipError_t launch_bwd(const CeArgs& a, hipStream_t stream) {
  if (a.V <= 64 * Piece<T>::N) return launch_bwd<T, 1, PAST>(a, stream);
  return launch_bwd<T, 4, PAST>(a, stream);
}

}  // namespace

size_t cross_entropy_uses(int64_t rows, int64_t V, bool f32) {
  if (rows <= 0 || !in_parts(rows, V, f32)) return 0;
  return (size_t)(rows_at_once(rows, V, f32) * parts_of(V, f32)) * sizeof(f32x4);
}

size_t cross_entropy_workspace(int64_t rows, int64_t V, bool f32) {
  // Not less for more rows than for fewer.
  return cross_entropy_uses(rows > kFewRows && !in_parts(rows, V, f32) ? kFewRows : rows, V, f32);
}

hipError_t launch_cross_entropy(const CeArgs& a, hipStream_t stream) {
  if (a.rows <= 0 || a.rows > INT32_MAX) return hipErrorInvalidValue;
  if (stream_activation(a.rows, a.V, a.f32))
    return a.f32 ? launch_loss<float, true>(a, stream) : launch_loss<uint16_t, true>(a, stream);
  return a.f32 ? launch_loss<float, false>(a, stream) : launch_loss<uint16_t, false>(a, stream);
}

hipError_t launch_cross_entropy_bwd(const CeArgs& a, hipStream_t stream) {
  if (stream_activation(a.rows, a.V, a.f32))
    return a.f32 ? launch_bwd<float, true>(a, stream) : launch_bwd<uint16_t, true>(a, stream);
  return a.f32 ? launch_bwd<float, false>(a, stream) : launch_bwd<uint16_t, false>(a, stream);
}

}  // namespace sppo
