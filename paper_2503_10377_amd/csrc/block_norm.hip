// The end of a transformer block in one pass: the norm after the block's
// branch, its gate, dropout, the scaled residual add and the norm in front of
// the next block; and the backward of all of it.
//   n = N_post(b);  h = alpha x + s keep (gate n);  z = N_pre(h)
// Done by separate kernels, n and h would travel to memory and back.  One row
// is held by a team of threads in registers (TEAM threads, PER groups of
// eight columns each); both norms' sums stay within the team.
#include <atomic>

#include "row_common.h"

namespace sppo {
namespace {

constexpr int kNone = 0, kLayer = 1, kRms = 2;
constexpr int kChannel = 1, kToken = 2;

// Has every cache line of the arguments fetched at once.  Their loads stand
// where the values are needed, and each first touch of a line is a trip to
// memory that the first rows would wait for, one after another: 0.4 us of a
// call (backward of 5001 x 1024 bf16 17.1 -> 16.6; nothing for the smaller
// arguments of dropout and the embedding).
__device__ __forceinline__ void fetch_args(const BlockNormArgs& a) {
  static_assert(sizeof(a) > 5 * 64 && sizeof(a) <= 6 * 64);
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&a);
  asm volatile("" ::"s"(w[0]), "s"(w[16]), "s"(w[32]), "s"(w[48]), "s"(w[64]), "s"(w[80]));
}

// A team's exchange of two moments: each wave's sum and squares, its number of
// columns and the inverse of that.
struct alignas(16) Moments {
  float s, q, n, inv;
};

// Fills the parts of the images that stay: the waves' columns.
template <int TEAM, int PER>
__device__ __forceinline__ void init_moments(Moments (*red)[TEAM / 64], int H, int tid) {
  if (tid < 2 * (TEAM / 64)) {
    const int w = tid >> 1;
    int n = 0;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int left = H - 8 * (64 * w + TEAM * p);
      n += left <= 0 ? 0 : (left < 512 ? left : 512);
    }
    red[tid & 1][w].n = (float)n;
    red[tid & 1][w].inv = n > 0 ? 1.f / n : 0.f;
  }
}

// Mean and 1 / sqrt(var + eps) of the row that the team holds in v.  Each wave
// takes the mean of its own columns and the squares around it; the waves'
// pairs are then joined (M2 = sum M2_w + n_w (mean_w - mean)^2), so one
// exchange serves both moments and nothing cancels.  red: one of the team's
// two images (written past the barrier that ended the reads of its last use).
template <int TEAM, int PER>
__device__ __forceinline__ void row_moments(const float (&v)[PER][8], int H, int tid, bool rms, float inv_h, float eps,
                                            Moments* red, float& mean, float& rstd) {
  constexpr int NW = TEAM / 64, LANES = TEAM < 64 ? TEAM : 64;
  float s = 0.f, q = 0.f, m = 0.f;
  if (!rms) {
#pragma unroll
    for (int p = 0; p < PER; ++p)
      if (8 * (tid + TEAM * p) < H) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[p][e];
      }
    s = lanes_sum<LANES>(s);
    m = s * (NW > 1 ? red[tid >> 6].inv : inv_h);
  }
#pragma unroll
  for (int p = 0; p < PER; ++p)
    if (8 * (tid + TEAM * p) < H) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = v[p][e] - m;
        q = fmaf(d, d, q);
      }
    }
  q = lanes_sum<LANES>(q);
  if constexpr (NW > 1) {
    if ((tid & 63) == 0) {
      red[tid >> 6].s = s;
      red[tid >> 6].q = q;
    }
    __syncthreads();
    Moments r[NW];
    s = q = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      r[w] = red[w];
      s += r[w].s;
    }
    m = s * inv_h;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float d = fmaf(-r[w].n, m, r[w].s);  // n_w (mean_w - mean); zero for RMS, whose sums are zero
      q += fmaf(d * r[w].inv, d, r[w].q);
    }
  }
  mean = m;
  rstd = __builtin_amdgcn_rsqf(fmaf(q, inv_h, eps));  // within an ulp
}

// Forward.  NT threads, teams of TEAM (the workgroup, one wave of it, or for
// narrow rows a half or a quarter of one).  A team takes rows in turn, so the
// parameters stay in its registers (read per row they would be 2.5 times the
// activations' bytes, out of L2), with a channel's gate folded into the norm
// after the branch: gate n = bh (gate gamma) + gate beta.  (Not an infinite
// one, which would leave 0 inf and inf - inf of sums that are neither: its sign
// is folded, and the sum multiplied after that.)  The next row's x and
// b are on their way while a row is worked on.  HBM-bound: 8192 x 4096 bf16
// with both LayerNorms, gate and dropout in 46 us, 5.8 TB/s (52.9 us and 5.1
// TB/s on new data every time), the vector units busy for 67% of it.
template <typename T, bool PAST, int NT, int TEAM, int PER>
__global__ __launch_bounds__(NT) void bn_fwd_kernel(BlockNormArgs a) {
  fetch_args(a);
  static_assert(TEAM == NT || TEAM <= 64, "");
  __shared__ Moments red[2][TEAM > 64 ? TEAM / 64 : 1];
  constexpr int TEAMS = NT / TEAM;
  const int H = a.H, tid = threadIdx.x % TEAM;
  const int64_t step = (int64_t)gridDim.x * TEAMS;
  // A row that belongs to whole waves is read and written as a buffer, so that
  // the next row's loads wait for none of this one's stores (3001 x 8192 with a
  // row's gate, which was read behind those loads: 41 -> 35 us).
  constexpr bool WAVE = TEAM >= 64;
  const int team = WAVE ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : threadIdx.x / TEAM;
  int64_t row = (int64_t)blockIdx.x * TEAMS + team;
  if (row >= a.rows) return;
  if constexpr (TEAM > 64) {
    init_moments<TEAM, PER>(red, H, tid);
    __syncthreads();
  }
  const Dropper drop(a.drop);
  const bool post = a.post != kNone, pre = a.pre != kNone;
  const bool token = a.gate_kind == kToken;
  const float inv_h = 1.f / H, scale = a.bscale * drop.scale;
  const int width = H * (int)sizeof(T);
  Eight<T> xn[PER], bn[PER];
  float gn = 1.f;  // the row's gate
  auto load = [&](int64_t r) {
    if constexpr (WAVE) {
      const int all = r < a.rows ? width : 0;
      const auto b = row_buffer(static_cast<const T*>(a.b) + r * a.ldb, all);
      const auto x = row_buffer(static_cast<const T*>(a.x) + r * a.ldx, all);
#pragma unroll
      for (int p = 0; p < PER; ++p) bn[p].template fetch<PAST>(b, 8 * (tid + TEAM * p));
#pragma unroll
      for (int p = 0; p < PER; ++p) xn[p].template fetch<PAST>(x, 8 * (tid + TEAM * p));
      gn = load_row4(row_buffer(a.gate + r, token && r < a.rows ? 4 : 0));
      return;
    }
    if (r >= a.rows) return;
    if (token) gn = a.gate[r];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int c = 8 * (tid + TEAM * p);
      if (c < H) {
        bn[p].template read<PAST>(static_cast<const T*>(a.b) + r * a.ldb + c);
        xn[p].template read<PAST>(static_cast<const T*>(a.x) + r * a.ldx + c);
      }
    }
  };
  load(row);  // on its way before the parameters
  float pg[PER][8], pb[PER][8], qg[PER][8], qb[PER][8];
  uint32_t endless = 0;  // bit 8 p + e: the channel's gate is infinite
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int c = 8 * (tid + TEAM * p);
#pragma unroll
    for (int e = 0; e < 8; ++e) pg[p][e] = 1.f, pb[p][e] = qg[p][e] = qb[p][e] = 0.f;
    if (c < H) {
      if (post) load8f(a.post_gamma + c, pg[p]);
      if (post && a.post_beta) load8f(a.post_beta + c, pb[p]);
      if (a.gate_kind == kChannel) {
        float g[8];
        load8f(a.gate + c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (__builtin_isinf(g[e])) {
            g[e] = copysignf(1.f, g[e]);
            endless |= 1u << (8 * p + e);
          }
          pg[p][e] *= g[e], pb[p][e] *= g[e];
        }
      }
      if (pre) load8f(a.pre_gamma + c, qg[p]);
      if (pre && a.pre_beta) load8f(a.pre_beta + c, qb[p]);
    }
  }
  const bool any_endless = __ballot(endless != 0) != 0;
  auto put_stats = [&](int kind, float* means, float* rstds, float mean, float rstd) {
    if constexpr (WAVE) {
      store_row4(row_buffer(means + row, kind == kLayer ? 4 : 0), tid == 0, mean);
      store_row4(row_buffer(rstds + row, kind != kNone ? 4 : 0), tid == 0, rstd);
    } else if (tid == 0) {
      if (kind == kLayer) means[row] = mean;
      if (kind != kNone) rstds[row] = rstd;
    }
  };
  auto put = [&](void* out, int64_t ld, bool on, int p, const float (&f)[8]) {
    T* o = static_cast<T*>(out) + row * ld;
    const int c = 8 * (tid + TEAM * p);
    if constexpr (WAVE) Eight<T>::template put<false>(row_buffer(o, on ? width : 0), c, f);
    else if (on && c < H) Eight<T>::store(o + c, f);
  };
  int ph = 0;
  for (; row < a.rows; row += step) {
    Eight<T> xr[PER];
    float v[PER][8];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      xr[p] = xn[p];
      bn[p].get(v[p]);
    }
    const float factor = token ? scale * gn : scale;
    load(row + step);
    float mean = 0.f, rstd = 1.f;
    if (post) {
      row_moments<TEAM, PER>(v, H, tid, a.post == kRms, inv_h, a.eps, red[ph], mean, rstd);
      ph ^= 1;
    }
    put_stats(a.post, a.post_mean, a.post_rstd, mean, rstd);
    const uint64_t g0 = (uint64_t)(a.drop.row0 + row) * (H / 8);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int c = 8 * (tid + TEAM * p);
      if (c < H) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[p][e] = factor * fmaf((v[p][e] - mean) * rstd, pg[p][e], pb[p][e]);
        if (any_endless) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (endless >> (8 * p + e) & 1) v[p][e] *= __builtin_inff();
        }
        drop.mask(g0 + c / 8, v[p]);
        float x[8];
        xr[p].get(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[p][e] = fmaf(a.alpha, x[e], v[p][e]);
      }
      put(a.h, a.ldh, true, p, v[p]);
    }
    if (pre) {
      row_moments<TEAM, PER>(v, H, tid, a.pre == kRms, inv_h, a.eps, red[ph], mean, rstd);
      ph ^= 1;
    }
    put_stats(a.pre, a.pre_mean, a.pre_rstd, mean, rstd);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] = fmaf((v[p][e] - mean) * rstd, qg[p][e], qb[p][e]);
      put(a.z, a.ldz, pre, p, v[p]);
    }
  }
}

// ------------------------------------------------------------------ backward
// With xh, bh the normalised h and b, m = s keep D, k = the row's gate (1
// unless the gate is per row) and the column sums over rows
//   S0 = sum dz xh, S1 = sum dz, S2 = sum k m bh, S3 = sum k m
// (no post norm: S2 = sum k m b), the parameter gradients are
//   dgamma_pre = S0, dbeta_pre = S1, dgamma_post = gate S2, dbeta_post = gate S3,
//   dgate (per channel) = gamma_post S2 + beta_post S3 (no post norm: S2),
// so the gate per channel needs no sum of its own.
struct Slots {
  bool on[4];
  int at[4];
  int n;
};
__host__ __device__ inline Slots bn_slots(const BlockNormArgs& a) {
  Slots s;
  const bool chan = a.gate_kind == kChannel && a.d_gate;
  s.on[0] = a.pre != kNone && a.d_pre_gamma;
  s.on[1] = a.pre != kNone && a.pre_beta && a.d_pre_beta;
  s.on[2] = chan || (a.post != kNone && a.d_post_gamma);
  s.on[3] = a.post != kNone && a.post_beta && (chan || a.d_post_beta);
  s.n = 0;
  for (int i = 0; i < 4; ++i) {
    s.at[i] = s.n;
    s.n += s.on[i];
  }
  return s;
}

// The team's sums of N values per thread, in every thread.
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], int tid, float* red) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_sum<TEAM < 64 ? TEAM : 64>(v[i]);
  if constexpr (TEAM > 64) {
    constexpr int NW = TEAM / 64;
    if ((tid & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) red[(tid >> 6) * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = red[i];
#pragma unroll
      for (int w = 1; w < NW; ++w) v[i] += red[w * N + i];
    }
  }
}

// A team takes rows in turn with the parameters in registers (gate and gamma
// as one) and the next row's h, dz, dh, b and statistics on their way, and adds
// its part of the column sums row by row.  8192 x 4096 bf16 with both
// LayerNorms, gate and dropout: 80 us and 5.7 for the sums' reduction, 5.2 TB/s
// with the column sums' traffic (through the caches 87 and 7, dx alone 3 of
// them).  MODE: what the branch needs beyond its mask (two waves a SIMD hold
// all of it in registers; asking for four, with some of it in scratch memory,
// doubled the time of the plain mode).
enum { kPlain = 0, kGated = 1, kNormed = 2 };
template <typename T, bool PAST, int MODE, int NT, int TEAM, int PER>
__global__ __launch_bounds__(NT) void bn_bwd_kernel(BlockNormArgs a) {
  fetch_args(a);
  constexpr bool POST = MODE == kNormed;
  constexpr int TEAMS = NT / TEAM;
  // the team's exchanges alternate between two images, as in the forward
  __shared__ float red_all[TEAM > 64 ? TEAMS : 1][2][TEAM > 64 ? 3 * (TEAM / 64) : 1];
  auto& red = red_all[TEAM > 64 ? threadIdx.x / TEAM : 0];
  constexpr bool AHEAD = sizeof(T) * PER <= 4;  // two groups of fp32 leave no registers for a row ahead
  // A row that belongs to whole waves is read and written as a buffer, so that
  // the next row's loads wait for none of this one's stores (5001 x 1024 16.6 ->
  // 15.9 us; without rows ahead 130 x 8192 fp32 would be 2 us slower).
  constexpr bool WAVE = TEAM >= 64 && AHEAD;
  const int H = a.H, tid = threadIdx.x % TEAM;
  const int team = WAVE ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : threadIdx.x / TEAM;
  const int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block;
  const int64_t r1 = r0 + a.rows_per_block < a.rows ? r0 + a.rows_per_block : a.rows;
  const Dropper drop(a.drop);
  const bool pre = a.pre != kNone;
  const float inv_h = 1.f / H, scale = a.bscale * drop.scale;
  Eight<T> hn[PER], bn[PER], zn[PER], dn[PER];
  float st[5] = {1.f, 0.f, 1.f, 0.f, 1.f};  // the row's statistics and gate
#pragma unroll
  for (int p = 0; p < PER; ++p) hn[p].zero(), bn[p].zero(), zn[p].zero(), dn[p].zero();
  auto load = [&](int64_t row) {
    if constexpr (WAVE) {
      const int one = row < r1 ? 4 : 0, all = row < r1 ? H * (int)sizeof(T) : 0;
      const auto h = row_buffer(static_cast<const T*>(a.h) + row * a.ldh, pre ? all : 0);
      const auto z = row_buffer(static_cast<const T*>(a.dz) + row * a.lddz, pre ? all : 0);
      const auto d = row_buffer(static_cast<const T*>(a.dh) + row * a.lddh, a.dh ? all : 0);
      const auto b = row_buffer(static_cast<const T*>(a.b) + row * a.ldb, a.b ? all : 0);
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int c = 8 * (tid + TEAM * p);
        hn[p].template fetch<PAST>(h, c);
        zn[p].template fetch<PAST>(z, c);
        dn[p].template fetch<PAST>(d, c);
        if constexpr (MODE != kPlain) bn[p].template fetch<PAST>(b, c);
      }
      st[0] = load_row4(row_buffer(a.pre_rstd + row, pre ? one : 0));
      st[1] = load_row4(row_buffer(a.pre_mean + row, a.pre == kLayer ? one : 0));
      if constexpr (POST) {
        st[2] = load_row4(row_buffer(a.post_rstd + row, one));
        st[3] = load_row4(row_buffer(a.post_mean + row, a.post == kLayer ? one : 0));
      }
      if constexpr (MODE != kPlain) st[4] = load_row4(row_buffer(a.gate + row, a.gate_kind == kToken ? one : 0));
      return;
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int c = 8 * (tid + TEAM * p);
      if (c < H) {
        if (pre) {
          hn[p].template read<PAST>(static_cast<const T*>(a.h) + row * a.ldh + c);
          zn[p].template read<PAST>(static_cast<const T*>(a.dz) + row * a.lddz + c);
        }
        if (a.dh) dn[p].template read<PAST>(static_cast<const T*>(a.dh) + row * a.lddh + c);
        if (MODE != kPlain && a.b) bn[p].template read<PAST>(static_cast<const T*>(a.b) + row * a.ldb + c);
      }
    }
    if (pre) st[0] = a.pre_rstd[row];
    if (a.pre == kLayer) st[1] = a.pre_mean[row];
    if (POST) st[2] = a.post_rstd[row];
    if (a.post == kLayer) st[3] = a.post_mean[row];
    if (MODE != kPlain && a.gate_kind == kToken) st[4] = a.gate[row];
  };
  int64_t row = r0 + team;
  if (WAVE || row < r1) load(row);  // on its way before the parameters
  float sum[4][PER][8], qg[PER][8], pg[PER][8];
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int c = 8 * (tid + TEAM * p);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pg[p][e] = 1.f;
      qg[p][e] = sum[0][p][e] = sum[1][p][e] = sum[2][p][e] = sum[3][p][e] = 0.f;
    }
    if (c < H) {
      if (pre) load8f(a.pre_gamma + c, qg[p]);
      if (POST) load8f(a.post_gamma + c, pg[p]);
      if (MODE != kPlain && a.gate_kind == kChannel) {
        float g[8];
        load8f(a.gate + c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) pg[p][e] *= g[e];
      }
    }
  }
  int ph = 0;
  // Teams of several waves meet at the workgroup's barriers: all go round as
  // often as the first (a team without a row has zeros).
  for (; TEAM > 64 && TEAMS > 1 ? row - team < r1 : row < r1; row += TEAMS) {
    const bool real = row < r1;
    Eight<T> hr[PER], br[PER], zr[PER];
    float D[PER][8];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      hr[p] = hn[p];
      br[p] = bn[p];
      zr[p] = zn[p];
      dn[p].get(D[p]);
    }
    const float rstd1 = st[0], mean1 = st[1], rstd = st[2], mean = st[3];
    const float k = a.gate_kind == kToken ? st[4] : 1.f;
    if (AHEAD && (WAVE || row + TEAMS < r1)) load(row + TEAMS);
    if (pre) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        if (8 * (tid + TEAM * p) < H) {
          float hv[8], zv[8];
          hr[p].get(hv);
          zr[p].get(zv);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float xh = (hv[e] - mean1) * rstd1, g = zv[e] * qg[p][e];
            s[0] += g;
            s[1] += g * xh;
            sum[0][p][e] += zv[e] * xh;
            sum[1][p][e] += zv[e];
          }
        }
      }
      team_sum<TEAM>(s, tid, red[ph]);
      ph ^= 1;
      const float m1 = a.pre == kLayer ? s[0] * inv_h : 0.f, m2 = s[1] * inv_h;
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        if (8 * (tid + TEAM * p) < H) {
          float hv[8], zv[8];
          hr[p].get(hv);
          zr[p].get(zv);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            D[p][e] += rstd1 * (fmaf(zv[e], qg[p][e], -m1) - (hv[e] - mean1) * rstd1 * m2);
        }
      }
    }
    const uint64_t g0 = (uint64_t)(a.drop.row0 + row) * (H / 8);
    const int all = real ? H * (int)sizeof(T) : 0;
    // dx (next read behind the branch's products, db by the first of them)
    auto put_dx = [&](int p) {
      const int c = 8 * (tid + TEAM * p);
      T* dx = static_cast<T*>(a.dx) + row * a.lddx;
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = a.alpha * D[p][e];
      if constexpr (WAVE) Eight<T>::template put<PAST>(row_buffer(dx, all), c, o);
      else if constexpr (PAST) Eight<T>::stream_out(dx + c, o);
      else Eight<T>::store(dx + c, o);
    };
    if constexpr (WAVE) {
#pragma unroll
      for (int p = 0; p < PER; ++p) put_dx(p);
    }
    float s[3] = {0.f, 0.f, 0.f};  // of w = m gamma gate_c, of w bh (no post norm: of m b), of m beta
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int c = 8 * (tid + TEAM * p);
      if (c < H) {
        if constexpr (!WAVE) put_dx(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) D[p][e] *= scale;
        drop.mask(g0 + c / 8, D[p]);
        if (a.gate_kind == kToken && POST && a.post_beta) {
          float bt[8];
          load8f(a.post_beta + c, bt);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[2] += D[p][e] * bt[e];
        }
        if constexpr (MODE != kPlain) {
          float bv[8];
          br[p].get(bv);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float m = D[p][e], bh = (bv[e] - mean) * rstd, w = m * pg[p][e];
            const float mb = POST || m != 0.f ? bh : 0.f;  // a dropped element is zero whatever b holds
            s[0] += w;
            s[1] += w * mb;
            sum[2][p][e] += (k * m) * mb;
            if (POST) sum[3][p][e] += k * m;
            D[p][e] = w;
          }
        }
      }
    }
    if (POST || (MODE == kGated && a.gate_kind == kToken)) {
      team_sum<TEAM>(s, tid, red[ph]);
      ph ^= 1;
    }
    if constexpr (MODE != kPlain && WAVE)
      store_row4(row_buffer(a.d_gate + row, a.gate_kind == kToken && a.d_gate && real ? 4 : 0), tid == 0, s[1] + s[2]);
    else if (MODE != kPlain && a.gate_kind == kToken && a.d_gate && tid == 0)
      a.d_gate[row] = s[1] + s[2];
    const float m1 = a.post == kLayer ? s[0] * inv_h : 0.f, m2 = s[1] * inv_h;
    const float kr = k * rstd;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int c = 8 * (tid + TEAM * p);
      if (c < H) {
        if constexpr (POST) {
          float bv[8];
          br[p].get(bv);
#pragma unroll
          for (int e = 0; e < 8; ++e) D[p][e] = kr * (D[p][e] - m1 - (bv[e] - mean) * rstd * m2);
        } else if constexpr (MODE == kGated) {
#pragma unroll
          for (int e = 0; e < 8; ++e) D[p][e] *= k;
        }
        if constexpr (!WAVE) Eight<T>::store(static_cast<T*>(a.db) + row * a.lddb + c, D[p]);
      }
      if constexpr (WAVE)
        Eight<T>::template put<false>(row_buffer(static_cast<T*>(a.db) + row * a.lddb, all), c, D[p]);
    }
    if (!AHEAD && row + TEAMS < r1) load(row + TEAMS);
  }
  // The workgroup's column sums: its teams' in team order.
  const Slots slots = bn_slots(a);
  float* part = a.part + (int64_t)blockIdx.x * slots.n * H;
  constexpr int SLOTS = 2 + MODE;  // S2 is of the gate or the norm after the branch, S3 of that norm
  if constexpr (TEAMS > 1) {
    __shared__ __attribute__((aligned(16))) float comb[SLOTS][TEAMS][8 * TEAM * PER];
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      if (!slots.on[i]) continue;
#pragma unroll
      for (int p = 0; p < PER; ++p) Eight<float>::store(&comb[i][team][8 * (tid + TEAM * p)], sum[i][p]);
    }
    __syncthreads();
    for (int c = 4 * threadIdx.x; c < H; c += 4 * NT) {
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) {
        if (!slots.on[i]) continue;
        f32x4 t = *reinterpret_cast<const f32x4*>(&comb[i][0][c]);
#pragma unroll
        for (int u = 1; u < TEAMS; ++u) t += *reinterpret_cast<const f32x4*>(&comb[i][u][c]);
        *reinterpret_cast<f32x4*>(part + slots.at[i] * H + c) = t;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      if (!slots.on[i]) continue;
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int c = 8 * (tid + TEAM * p);
        if (c < H) Eight<float>::store(part + slots.at[i] * H + c, sum[i][p]);
      }
    }
  }
}

// The column sums over the workgroups, and the gradients made from them.  A
// workgroup covers 32 columns, with 256 threads for each sum that is needed:
// 32 groups of rows, group t adding blocks t, t + 32, ... in order (the loads
// all at once: 256 blocks of 1024 columns and two sums in 3.9 us, one load after
// another 1.3 us more), then the groups are added pairwise.
constexpr int kRedCols = 32, kRedGroups = 32, kRedThreads = kRedCols / 4 * kRedGroups;
constexpr int kRedAhead = 8;  // 256 blocks at once
template <bool ADD>
__global__ __launch_bounds__(4 * kRedThreads) void bn_reduce_kernel(BlockNormArgs a) {
  fetch_args(a);
  __shared__ __attribute__((aligned(16))) float red[4][kRedGroups][kRedCols + 4];
  __shared__ float total[4][kRedCols];
  const int i = threadIdx.x / kRedThreads, th = threadIdx.x % kRedThreads;
  const int lc = th % (kRedCols / 4) * 4, t = th / (kRedCols / 4);
  const int c = blockIdx.x * kRedCols + lc, H = a.H;
  const Slots slots = bn_slots(a);
  const int64_t step = (int64_t)slots.n * H;
  const bool post = a.post != kNone, chan = a.gate_kind == kChannel;
  const int oc = blockIdx.x * kRedCols + threadIdx.x;
  // what the gradients are made with and added to, on its way before the sums
  const int at = threadIdx.x < kRedCols && oc < H ? oc : 0;
  const float gate = chan ? a.gate[at] : 1.f;
  const float gamma = chan && post ? a.post_gamma[at] : 1.f;
  const float beta = chan && post && a.post_beta ? a.post_beta[at] : 0.f;
  float* const out[5] = {slots.on[0] ? a.d_pre_gamma : nullptr, slots.on[1] ? a.d_pre_beta : nullptr,
                         post ? a.d_post_gamma : nullptr, post && a.post_beta ? a.d_post_beta : nullptr,
                         chan ? a.d_gate : nullptr};
  float old[5];
#pragma unroll
  for (int u = 0; u < 5; ++u) {
    old[u] = 0.f;
    if (ADD && out[u]) old[u] = out[u][at];
  }
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c < H) {
    const float* p = a.part + (int64_t)i * H + c;
    for (int b0 = t; b0 < a.nblocks; b0 += kRedAhead * kRedGroups) {
      f32x4 v[kRedAhead];
#pragma unroll
      for (int u = 0; u < kRedAhead; ++u) {
        const int b = b0 + kRedGroups * u;
        v[u] = *reinterpret_cast<const f32x4*>(p + (b < a.nblocks ? b : b0) * step);
      }
#pragma unroll
      for (int u = 0; u < kRedAhead; ++u)
        if (b0 + kRedGroups * u < a.nblocks) s += v[u];
    }
  }
  *reinterpret_cast<f32x4*>(&red[i][t][lc]) = s;
  __syncthreads();
  if (th < kRedCols) {
    float v[kRedGroups];
#pragma unroll
    for (int u = 0; u < kRedGroups; ++u) v[u] = red[i][u][th];
#pragma unroll
    for (int n = kRedGroups / 2; n > 0; n /= 2) {
#pragma unroll
      for (int u = 0; u < n; ++u) v[u] += v[u + n];
    }
    total[i][th] = v[0];
  }
  __syncthreads();
  if (threadIdx.x >= kRedCols || oc >= H) return;
  float S[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) S[u] = slots.on[u] ? total[slots.at[u]][threadIdx.x] : 0.f;
  const float sums[5] = {S[0], S[1], gate * S[2], gate * S[3], fmaf(beta, S[3], gamma * S[2])};
#pragma unroll
  for (int u = 0; u < 5; ++u)
    if (out[u]) out[u][oc] = ADD ? old[u] + sums[u] : sums[u];
}

template <typename T, bool PAST, int NT, int TEAM, int PER>
hipError_t fwd(const BlockNormArgs& a, hipStream_t stream) {
  const int64_t teams = NT / TEAM, all = (a.rows + teams - 1) / teams;
  // As many workgroups as are resident at once: more would begin when the first
  // have taken all of their rows (8192 x 4096: 768 of them 52.8 us, 1024 57.1).
  // Asked for until it is known: a query that fails is the call's error, and the
  // next call asks again.
  static std::atomic<int> known{0};
  int resident = known.load(std::memory_order_relaxed);
  if (resident == 0) {
    const hipError_t e =
        hipOccupancyMaxActiveBlocksPerMultiprocessor(&resident, bn_fwd_kernel<T, PAST, NT, TEAM, PER>, NT, 0);
    if (e != hipSuccess) {
      (void)hipGetLastError();  // reported here, not by the next launch
      return e;
    }
    if (resident < 1) return hipErrorLaunchOutOfResources;
    known.store(resident, std::memory_order_relaxed);
  }
  const int64_t most = (int64_t)device_cus() * resident;
  hipLaunchKernelGGL((bn_fwd_kernel<T, PAST, NT, TEAM, PER>), dim3((unsigned)(all < most ? all : most)), dim3(NT), 0,
                     stream, a);
  return hipGetLastError();
}

template <typename T, bool PAST, int NT, int TEAM, int PER>
hipError_t bwd(const BlockNormArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.nblocks), block(NT);
  if (a.post != kNone)
    hipLaunchKernelGGL((bn_bwd_kernel<T, PAST, kNormed, NT, TEAM, PER>), grid, block, 0, stream, a);
  else if (a.gate_kind != kNone)
    hipLaunchKernelGGL((bn_bwd_kernel<T, PAST, kGated, NT, TEAM, PER>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((bn_bwd_kernel<T, PAST, kPlain, NT, TEAM, PER>), grid, block, 0, stream, a);
  return hipGetLastError();
}

// bf16 rows take two groups of eight columns a thread where they can: what a
// wave does once per row (its share of the sums, the statistics) is half as
// much per element (forward of 8192 x 4096 with one: 88 us).  fp32 rows have
// twice the bytes and twice the registers per element; rows of up to 6 x 512
// columns take six waves (6553 x 2560 on new data: eight waves 60 us, six 57; for
// bf16 rows two groups in four waves 32, one in six 44).
template <typename T, bool PAST>
hipError_t forward(const BlockNormArgs& a, hipStream_t stream) {
  constexpr int P = sizeof(T) == 2 ? 2 : 1;
  if (a.H <= 128) return fwd<T, PAST, 256, 16, 1>(a, stream);
  if (a.H <= 256) return fwd<T, PAST, 256, 32, 1>(a, stream);
  if (a.H <= 512) return fwd<T, PAST, 256, 64, 1>(a, stream);
  if (a.H <= 1024) return fwd<T, PAST, 256, 64, 2>(a, stream);
  if (a.H <= 2048) return fwd<T, PAST, 256 / P, 256 / P, P>(a, stream);
  if constexpr (P == 1)
    if (a.H <= 6 * 512) return fwd<T, PAST, 384, 384, 1>(a, stream);
  if (a.H <= 4096) return fwd<T, PAST, 512 / P, 512 / P, P>(a, stream);
  return fwd<T, PAST, 512, 512, 2>(a, stream);  // 1024 threads would have 128 registers each, too few
}

// The backward's workgroups hold as many teams as fit 512 threads, one
// workgroup a compute unit, so that few of them leave column sums (8192 x 4096
// through the caches, with 512 workgroups of one team: 100 us with the sums'
// reduction, with 256 of two teams 94); up to 512 columns a wave needs fewer registers and twice as
// many fit.
// Widths that would leave waves of such a team half empty take one group a
// thread and, with fewer registers, 768 threads (with LayerNorms, gate and
// dropout on new data, two groups in 512 threads against this: 13107 x 1280 bf16
// 63 and 55 us, 6553 x 2560 60.5 and 55, 3276 x 5120 59.7 and 57; 6553 x 2560
// fp32 102 and 99).
template <typename T, bool PAST>
hipError_t backward(const BlockNormArgs& a, hipStream_t stream) {
  constexpr int P = sizeof(T) == 2 ? 2 : 1;
  if (a.H <= 128) return bwd<T, PAST, 256, 16, 1>(a, stream);
  if (a.H <= 256) return bwd<T, PAST, 256, 32, 1>(a, stream);
  if (a.H <= 512) return bwd<T, PAST, 256, 64, 1>(a, stream);
  if (a.H <= 1024) return bwd<T, PAST, 512, 64, 2>(a, stream);
  if constexpr (P == 2) {
    if (a.H <= 3 * 512) return bwd<T, PAST, 768, 192, 1>(a, stream);
    if (a.H > 8 * 512 && a.H <= 12 * 512) return bwd<T, PAST, 768, 768, 1>(a, stream);
  }
  if (a.H <= 2048) return bwd<T, PAST, 512, 256 / P, P>(a, stream);
  if (a.H <= 6 * 512) return bwd<T, PAST, 768, 384, 1>(a, stream);
  if (a.H <= 4096) return bwd<T, PAST, 512, 512 / P, P>(a, stream);
  return bwd<T, PAST, 512, 512, 2>(a, stream);
}

// Teams of a workgroup of the backward (as dispatched above), and the most
// workgroups a number of rows takes.
int teams_of(int H, int f32) {
  if (H <= 512) return H <= 128 ? 16 : H <= 256 ? 8 : 4;
  if (H <= 1024) return 8;
  if (H <= 2048) return f32 ? 2 : 4;
  if (H <= 6 * 512) return 2;
  return H <= 4096 && !f32 ? 2 : 1;
}
int64_t bwd_blocks(int64_t rows, int H, int f32) {
  const int64_t teams = teams_of(H, f32), groups = (rows + teams - 1) / teams, most = H <= 512 ? 512 : 256;
  return groups < most ? groups : most;
}

}  // namespace

size_t block_norm_bwd_workspace(const BlockNormArgs& a) {
  // as if every gradient were wanted
  BlockNormArgs b = a;
  float any;
  b.d_post_gamma = b.d_post_beta = b.d_gate = b.d_pre_gamma = b.d_pre_beta = &any;
  return (size_t)bwd_blocks(a.rows, a.H, a.f32) * bn_slots(b).n * (size_t)a.H * sizeof(float);
}

hipError_t launch_block_norm_fwd(const BlockNormArgs& a, hipStream_t stream) {
  if (a.rows <= 0 || a.H <= 0 || a.H % 8 || a.H > kBnMaxH) return hipErrorInvalidValue;
  if (stream_activation(a.rows, a.H, a.f32))
    return a.f32 ? forward<float, true>(a, stream) : forward<uint16_t, true>(a, stream);
  return a.f32 ? forward<float, false>(a, stream) : forward<uint16_t, false>(a, stream);
}

hipError_t launch_block_norm_bwd(const BlockNormArgs& a, hipStream_t stream) {
  if (a.rows <= 0 || a.H <= 0 || a.H % 8 || a.H > kBnMaxH) return hipErrorInvalidValue;
  BlockNormArgs b = a;
  const int64_t teams = teams_of(a.H, a.f32), most = bwd_blocks(a.rows, a.H, a.f32);
  b.rows_per_block = (int)((a.rows + most * teams - 1) / (most * teams) * teams);
  b.nblocks = (int)((a.rows + b.rows_per_block - 1) / b.rows_per_block);
  const bool past = stream_activation(a.rows, a.H, a.f32);
  const hipError_t e = past ? (a.f32 ? backward<float, true>(b, stream) : backward<uint16_t, true>(b, stream))
                            : (a.f32 ? backward<float, false>(b, stream) : backward<uint16_t, false>(b, stream));
  const int sums = bn_slots(a).n;
  if (e != hipSuccess || sums == 0) return e;
  const dim3 grid((unsigned)((a.H + kRedCols - 1) / kRedCols)), block((unsigned)(sums * kRedThreads));
  if (a.accumulate)
    hipLaunchKernelGGL(bn_reduce_kernel<true>, grid, block, 0, stream, b);
  else
    hipLaunchKernelGGL(bn_reduce_kernel<false>, grid, block, 0, stream, b);
  return hipGetLastError();
}

}  // namespace sppo
