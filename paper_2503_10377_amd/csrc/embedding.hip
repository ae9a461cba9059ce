// Token embedding with scale and dropout, and the gradient of its table.
//
// Forward: y[r] = drop(scale table[id_r]), one pass over y; HBM-bound.
//
// Backward: dtable[v] (+)= scale sum_{r: id_r = v} drop(dy[r]).  Rows of a
// token lie anywhere and a frequent token has thousands of them, so the rows
// are first sorted by token (stable: rows of a token stay in order), then cut
// into tiles of kTile sorted rows that sum the runs of equal tokens they hold.
// A run inside one tile goes to the table at once; of a run that crosses
// tiles each tile leaves a partial sum, and a last kernel adds these in tile
// order.  No atomics: every sum has a fixed order.
#include "row_common.h"

namespace sppo {
namespace {

constexpr int kThreads = 256, kUnroll = 4;
constexpr int64_t kMaxGroups = (int64_t)1 << 30;  // of a launch: below fast_div's 2^31

// The token of row r as an index below V, or V if it lies outside the table
// (compared as 64-bit numbers: an id past 32 bits is outside).
__device__ __forceinline__ uint32_t token(const void* ids, int id64, int64_t r, int64_t V) {
  const int64_t id = id64 ? static_cast<const int64_t*>(ids)[r] : static_cast<const int32_t*>(ids)[r];
  return (uint32_t)(id >= 0 && id < V ? id : V);
}

// A thread takes kUnroll groups of eight elements, 256 groups apart.
template <typename T>
__global__ __launch_bounds__(kThreads) void embed_fwd_kernel(EmbedArgs a, FastDiv per_row, uint32_t groups) {
  const Dropper drop(a.drop);
  const uint32_t cpr = (uint32_t)a.H / 8;
  const uint64_t g0 = (uint64_t)a.drop.row0 * cpr;
  Eight<T> x[kUnroll];
  uint32_t g[kUnroll], row[kUnroll], col[kUnroll], id[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    g[u] = blockIdx.x * (kThreads * kUnroll) + kThreads * u + threadIdx.x;
    if (g[u] >= groups) continue;
    row[u] = fast_div(g[u], per_row);
    col[u] = (g[u] - row[u] * cpr) * 8;
    id[u] = token(a.ids, a.id64, row[u], a.V);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (g[u] >= groups) continue;
    x[u].zero();
    if (id[u] < a.V) x[u].load(static_cast<const T*>(a.table) + (int64_t)id[u] * a.ldt + col[u]);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (g[u] >= groups) continue;
    float f[8];
    x[u].get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = id[u] < a.V ? f[e] * a.scale : 0.f;  // zero also where scale is not finite
    drop.apply(g0 + g[u], f);
    Eight<T>::store(static_cast<T*>(a.y) + (int64_t)row[u] * a.ldy + col[u], f);
  }
}

// ------------------------------------------------------------------ the sort
// Least significant digit first, up to kMaxDigitBits bits a pass.  The keys
// are cut into at most kMaxSortTiles tiles, one workgroup each; a pass counts
// each tile's digits (sort_count), then every workgroup finds where its keys
// of each digit go from all the counts, and moves its keys (sort_scatter).
constexpr int kMaxDigitBits = 9, kMaxDigits = 1 << kMaxDigitBits;
constexpr int kMaxSortTiles = 128;
constexpr int kSortThreads = 512, kSortKeys = 2, kSortWaves = kSortThreads / 64;
constexpr int kSortStep = kSortThreads * kSortKeys;  // keys a workgroup handles at a time

struct SortArgs {
  int64_t n;
  int tiles;
  int64_t per_tile;     // a multiple of kSortStep
  const uint32_t* key;  // previous pass; NULL: the tokens themselves, row r at place r
  const uint32_t* row;
  uint32_t* key_out;
  uint32_t* row_out;
  uint32_t* counts;     // [tiles][1 << bits]
  int shift, bits;
  const void* ids;
  int id64;
  int64_t V;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs& s, int64_t i) {
  return s.key ? s.key[i] : token(s.ids, s.id64, i, s.V);
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs s) {
  __shared__ uint32_t cnt[kMaxDigits];
  const int digits = 1 << s.bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) cnt[d] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * s.per_tile;
  const int64_t i1 = i0 + s.per_tile < s.n ? i0 + s.per_tile : s.n;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortThreads)
    atomicAdd(&cnt[(sort_key(s, i) >> s.shift) & (digits - 1)], 1u);  // counts: any order gives the same
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) s.counts[(int64_t)blockIdx.x * digits + d] = cnt[d];
}

__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortArgs s) {
  __shared__ uint32_t base[kMaxDigits];             // next place of each digit of this tile
  __shared__ uint32_t cnt[kSortWaves][kMaxDigits];  // keys of each digit in a wave, then their first place
  __shared__ uint32_t wsum[kSortWaves];
  const int digits = 1 << s.bits, tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  static_assert(kSortThreads >= kMaxDigits, "a thread per digit");
  // Digit d's keys of this tile start after all keys of smaller digits and
  // those of digit d in earlier tiles.
  uint32_t all = 0, before = 0;
  if (tid < digits) {
#pragma unroll 8
    for (int t = 0; t < s.tiles; ++t) {
      const uint32_t c = s.counts[(int64_t)t * digits + tid];
      all += c;
      if (t < (int)blockIdx.x) before += c;
    }
  }
  uint32_t incl = all;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t v = __shfl_up(incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  uint32_t off = incl - all;
  for (int u = 0; u < w; ++u) off += wsum[u];
  if (tid < digits) base[tid] = off + before;
  const int64_t i0 = (int64_t)blockIdx.x * s.per_tile;
  const int64_t i1 = i0 + s.per_tile < s.n ? i0 + s.per_tile : s.n;
  for (int64_t step = i0; step < i1; step += kSortStep) {
#pragma unroll
    for (int u = 0; u < kSortWaves; ++u)
      if (tid < digits) cnt[u][tid] = 0;
    __syncthreads();
    // A wave holds kSortKeys times 64 consecutive keys; a key's rank among
    // the wave's keys of its digit: those of earlier rounds (the counter),
    // and the lanes below with the same digit.
    uint32_t key[kSortKeys], row[kSortKeys], rank[kSortKeys];
#pragma unroll
    for (int u = 0; u < kSortKeys; ++u) {
      const int64_t i = step + (w * kSortKeys + u) * 64 + lane;
      const bool in = i < i1;
      key[u] = in ? sort_key(s, i) : 0;
      row[u] = in ? (s.key ? s.row[i] : (uint32_t)i) : 0;
      const uint32_t d = (key[u] >> s.shift) & (digits - 1);
      uint64_t same = __ballot(in);
      for (int b = 0; b < s.bits; ++b) {
        const uint64_t ones = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? ones : ~ones;
      }
      const int first = in ? __ffsll((unsigned long long)same) - 1 : lane;
      uint32_t old = 0;
      if (in && lane == first) old = atomicAdd(&cnt[w][d], (uint32_t)__popcll(same));
      old = __shfl(old, first);
      rank[u] = old + __popcll(same & (((uint64_t)1 << lane) - 1));
    }
    __syncthreads();
    if (tid < digits) {
      uint32_t at = base[tid];
#pragma unroll
      for (int u = 0; u < kSortWaves; ++u) {
        const uint32_t c = cnt[u][tid];
        cnt[u][tid] = at;
        at += c;
      }
      base[tid] = at;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSortKeys; ++u) {
      const int64_t i = step + (w * kSortKeys + u) * 64 + lane;
      if (i < i1) {
        const uint32_t at = cnt[w][(key[u] >> s.shift) & (digits - 1)] + rank[u];
        s.key_out[at] = key[u];
        s.row_out[at] = row[u];
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ the sums
constexpr int kTile = 32;  // sorted rows of a workgroup
constexpr int kSlab = kThreads * 8;  // columns of a workgroup

struct SumArgs {
  int64_t n;
  const uint32_t* key;  // sorted tokens (outside the table: V, at the end)
  const uint32_t* row;
  float* part;          // [tiles][2][H]: the run that enters the tile, the run that leaves it
};

__global__ __launch_bounds__(256) void embed_zero_kernel(EmbedArgs a) {
  for (int64_t v = blockIdx.x; v < a.V; v += gridDim.x)
    for (int c = 4 * threadIdx.x; c < a.H; c += 1024)
      *reinterpret_cast<f32x4*>(a.dtable + v * a.lddt + c) = f32x4{0.f, 0.f, 0.f, 0.f};
}

template <typename T>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(EmbedArgs a, SumArgs s) {
  const int c = blockIdx.y * kSlab + 8 * threadIdx.x;
  if (c >= a.H) return;
  const int64_t i0 = (int64_t)blockIdx.x * kTile, i1 = i0 + kTile < s.n ? i0 + kTile : s.n;
  const Dropper drop(a.drop);
  const uint32_t V = (uint32_t)a.V;
  const uint32_t prev = i0 > 0 ? s.key[i0 - 1] : V;  // V: no run enters
  const uint32_t next = i1 < s.n ? s.key[i1] : V;    // V: no run leaves
  uint32_t cur = s.key[i0];
  bool entered = cur == prev;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto flush = [&](bool leaves) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= a.scale;
    if (entered || leaves) {
      Eight<float>::store(s.part + ((int64_t)blockIdx.x * 2 + (entered ? 0 : 1)) * a.H + c, acc);
    } else {
      float* out = a.dtable + (int64_t)cur * a.lddt + c;
      if (a.accumulate) {
        float o[8];
        load8f(out, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += o[e];
      }
      Eight<float>::store(out, acc);
    }
  };
  for (int64_t i = i0; i < i1; ++i) {
    const uint32_t k = s.key[i];
    if (k != cur) {
      flush(false);
      cur = k;
      entered = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    }
    if (k >= V) return;
    const uint32_t r = s.row[i];
    Eight<T> x;
    x.load(static_cast<const T*>(a.dy) + (int64_t)r * a.ldy + c);
    float f[8];
    x.get(f);
    drop.apply((uint64_t)(a.drop.row0 + r) * (a.H / 8) + c / 8, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += f[e];
  }
  flush(cur == next);
}

// The run that leaves tile t (if one begins there): its partial sums, from
// tile t's second and the following tiles' first, in tile order.
constexpr int kJoinCols = 256, kJoinGroups = 4;
__global__ __launch_bounds__(kJoinCols / 4 * kJoinGroups) void embed_join_kernel(EmbedArgs a, SumArgs s) {
  __shared__ __attribute__((aligned(16))) float red[kJoinGroups][kJoinCols];
  const int64_t t = blockIdx.x, i0 = t * kTile, last = i0 + kTile - 1;
  if (last + 1 >= s.n) return;
  const uint32_t k = s.key[last], V = (uint32_t)a.V;
  if (k >= V || s.key[last + 1] != k) return;
  if (s.key[i0] == k && i0 > 0 && s.key[i0 - 1] == k) return;  // it began before this tile
  // the last tile the run reaches: the last place whose key is k
  int64_t lo = last + 1, hi = s.n;  // key[lo] == k; key[hi] > k, or the end
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if (s.key[mid] == k) lo = mid;
    else hi = mid;
  }
  const int64_t end = lo / kTile;
  const int lc = threadIdx.x % (kJoinCols / 4) * 4, grp = threadIdx.x / (kJoinCols / 4);
  const int c = blockIdx.y * kJoinCols + lc;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (c < a.H) {
#pragma unroll 4
    for (int64_t u = t + grp; u <= end; u += kJoinGroups)
      sum += *reinterpret_cast<const f32x4*>(s.part + (u * 2 + (u == t ? 1 : 0)) * a.H + c);
  }
  *reinterpret_cast<f32x4*>(&red[grp][lc]) = sum;
  __syncthreads();
  if (grp == 0 && c < a.H) {
#pragma unroll
    for (int u = 1; u < kJoinGroups; ++u) sum += *reinterpret_cast<const f32x4*>(&red[u][lc]);
    f32x4* out = reinterpret_cast<f32x4*>(a.dtable + (int64_t)k * a.lddt + c);
    if (a.accumulate) sum += *out;
    *out = sum;
  }
}

// ------------------------------------------------------------------ the plan
struct Plan {
  int64_t tiles;  // of the sums
  int64_t keys, counts, part, bytes;  // byte offsets: four arrays of n words from 0, then these
};
Plan plan(int64_t rows, int H) {
  Plan p;
  p.tiles = (rows + kTile - 1) / kTile;
  p.keys = (rows * 4 + 255) / 256 * 256;
  p.counts = 4 * p.keys;
  p.part = p.counts + (int64_t)kMaxSortTiles * kMaxDigits * 4;
  p.bytes = p.part + p.tiles * 2 * (int64_t)H * 4;
  return p;
}

template <typename T>
hipError_t forward(const EmbedArgs& a, hipStream_t stream) {
  const int64_t cpr = a.H / 8, rows_per = kMaxGroups / cpr;
  const FastDiv div = fast_divisor((uint32_t)cpr);
  for (int64_t r = 0; r < a.rows; r += rows_per) {
    EmbedArgs b = a;
    b.rows = a.rows - r < rows_per ? a.rows - r : rows_per;
    b.ids = static_cast<const char*>(a.ids) + r * (a.id64 ? 8 : 4);
    b.y = static_cast<T*>(a.y) + r * a.ldy;
    b.drop.row0 += r;
    const uint32_t groups = (uint32_t)(b.rows * cpr);
    hipLaunchKernelGGL(embed_fwd_kernel<T>, dim3((groups + kThreads * kUnroll - 1) / (kThreads * kUnroll)),
                       dim3(kThreads), 0, stream, b, div, groups);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t backward(const EmbedArgs& a, hipStream_t stream) {
  const Plan p = plan(a.rows, a.H);
  char* ws = static_cast<char*>(a.workspace);
  uint32_t* arr[4];
  for (int i = 0; i < 4; ++i) arr[i] = reinterpret_cast<uint32_t*>(ws + i * p.keys);
  int bits = 1;
  while (((int64_t)1 << bits) <= a.V) ++bits;  // keys 0 .. V
  const int passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
  SortArgs s{};
  s.n = a.rows;
  s.per_tile = (a.rows + (int64_t)kMaxSortTiles * kSortStep - 1) / ((int64_t)kMaxSortTiles * kSortStep) * kSortStep;
  s.tiles = (int)((a.rows + s.per_tile - 1) / s.per_tile);
  s.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
  s.ids = a.ids;
  s.id64 = a.id64;
  s.V = a.V;
  hipError_t e;
  if (!a.accumulate) {
    hipLaunchKernelGGL(embed_zero_kernel, dim3((unsigned)(a.V < 65536 ? a.V : 65536)), dim3(256), 0, stream, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  for (int i = 0, at = 0; i < passes; ++i) {
    s.shift = at;
    s.bits = (bits - at + passes - i - 1) / (passes - i);
    at += s.bits;
    s.key_out = arr[2 * (i & 1)];
    s.row_out = arr[2 * (i & 1) + 1];
    hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)s.tiles), dim3(kSortThreads), 0, stream, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(sort_scatter_kernel, dim3((unsigned)s.tiles), dim3(kSortThreads), 0, stream, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    s.key = s.key_out;
    s.row = s.row_out;
  }
  SumArgs u{a.rows, s.key, s.row, reinterpret_cast<float*>(ws + p.part)};
  hipLaunchKernelGGL(embed_sum_kernel<T>, dim3((unsigned)p.tiles, (unsigned)((a.H + kSlab - 1) / kSlab)),
                     dim3(kThreads), 0, stream, a, u);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)p.tiles, (unsigned)((a.H + kJoinCols - 1) / kJoinCols)),
                     dim3(kJoinCols / 4 * kJoinGroups), 0, stream, a, u);
  return hipGetLastError();
}

}  // namespace

size_t embedding_workspace(int64_t rows, int H) { return (size_t)plan(rows, H).bytes; }

hipError_t launch_embedding_fwd(const EmbedArgs& a, hipStream_t stream) {
  if (a.rows <= 0 || a.H <= 0 || a.H % 8) return hipErrorInvalidValue;
  return a.f32 ? forward<float>(a, stream) : forward<uint16_t>(a, stream);
}

hipError_t launch_embedding_bwd(const EmbedArgs& a, hipStream_t stream) {
  if (a.rows <= 0 || a.H <= 0 || a.H % 8) return hipErrorInvalidValue;
  return a.f32 ? backward<float>(a, stream) : backward<uint16_t>(a, stream);
}

}  // namespace sppo
