// Token embedding with scale and dropout, and the gradient of its table.
//
// Forward: y[r] = drop(scale table[id_r]), one pass over y; HBM-bound.
//
// Backward: dtable[v] (+)= scale sum_{r: id_r = v} drop(dy[r]).  Rows of a
// token lie anywhere and a frequent token has thousands of them, so the rows
// are first sorted by token (rows of a token stay in order), then waves sum 16
// sorted rows each, run by run of equal tokens.  A short run goes to the table
// at once; of a long one the waves leave partial sums, which are added in the
// order of the rows.  Every sum has a fixed order, so the gradient has the same
// bits every time.  A few rows take a kernel that needs no sorted list.
#include "row_common.h"

namespace sppo {
namespace {

constexpr int kThreads = 256, kUnroll = 4;
constexpr int64_t kMaxGroups = (int64_t)1 << 30;  // of a launch: below fast_div's 2^31

// A token as an index below V, or V if it lies outside the table (compared as
// 64-bit numbers: an id past 32 bits is outside).
__device__ __forceinline__ uint32_t inside(int64_t id, int64_t V) { return (uint32_t)(id >= 0 && id < V ? id : V); }

// A thread takes kUnroll groups of eight elements, 256 groups apart: the ids
// first, then the table's pieces, then the draws (19 us of the vector units for
// 8192 x 4096 bf16, beside 16 for its bytes at 6.0 TB/s: 22.2 us on new tokens
// every time; with branches around the loads 25).
template <typename T>
__global__ __launch_bounds__(kThreads) void embed_fwd_kernel(EmbedArgs a, FastDiv per_row, uint32_t groups) {
  const Dropper drop(a.drop);
  const uint32_t cpr = (uint32_t)a.H / 8;
  const uint64_t g0 = (uint64_t)a.drop.row0 * cpr;
  const float scale = a.scale * drop.scale;  // finite: a row of zeros stays one
  // No branches around the loads (a thread past the end takes the last group
  // again, an id outside the table reads its row 0), so that none waits for
  // another; the draws come before the pieces are waited for.
  Eight<T> x[kUnroll];
  uint32_t g[kUnroll], row[kUnroll], col[kUnroll], id[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const uint32_t i = blockIdx.x * (kThreads * kUnroll) + kThreads * u + threadIdx.x;
    g[u] = i < groups ? i : groups - 1;
    row[u] = fast_div(g[u], per_row);
    col[u] = (g[u] - row[u] * cpr) * 8;
  }
  if (a.id64) {
    int64_t v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) v[u] = static_cast<const int64_t*>(a.ids)[row[u]];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) id[u] = inside(v[u], a.V);
  } else {
    int32_t v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) v[u] = static_cast<const int32_t*>(a.ids)[row[u]];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) id[u] = inside(v[u], a.V);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    x[u].load(static_cast<const T*>(a.table) + (int64_t)(id[u] < a.V ? id[u] : 0) * a.ldt + col[u]);
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    u32x4 w;
    if (drop.t16) w = drop.draw(g0 + g[u]);
    float f[8];
    if (id[u] >= a.V) x[u].zero();
    x[u].get(f);
    if (drop.t16) drop.keep(w, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= scale;
    if (blockIdx.x * (kThreads * kUnroll) + kThreads * u + threadIdx.x < groups)
      Eight<T>::store(static_cast<T*>(a.y) + (int64_t)row[u] * a.ldy + col[u], f);
  }
}

// ------------------------------------------------------------------ zeros
// Overwriting starts from a table of zeros (rows with tokens are written
// again later).  The fill is the largest stream of bytes of the backward and
// nothing before the sums needs it, so it rides along with the sort: the sort's
// few workgroups come first in each launch, the others clear a part of the table.
struct ZeroArgs {
  float* table;
  int64_t ld, v0, v1;  // rows [v0, v1)
  int H;
};

// The share of block `block` of `blocks`, in pieces of 16 bytes.
template <int NT>
__device__ __forceinline__ void zero_rows(const ZeroArgs& z, int64_t block, int64_t blocks) {
  const int64_t per_row = z.H / 4, stride = blocks * NT;
  const int64_t dr = stride / per_row, dc = stride - dr * per_row, i = block * NT + threadIdx.x;
  int64_t r = i / per_row, c = i - r * per_row;
  for (r += z.v0; r < z.v1; r += dr, c += dc) {
    if (c >= per_row) {
      c -= per_row;
      if (++r >= z.v1) return;
    }
    *reinterpret_cast<f32x4*>(z.table + r * z.ld + 4 * c) = f32x4{0.f, 0.f, 0.f, 0.f};
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
constexpr int kScan = 32;                            // tiles whose counts are on their way at once

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

// Keys (and rows) i[u] of a pass, those from `end` on as the first one's:
// without branches between the loads, so all are on their way at once.
template <int N>
__device__ __forceinline__ void sort_keys(const SortArgs& s, const int64_t (&i)[N], int64_t end, uint32_t (&key)[N],
                                          uint32_t (&row)[N]) {
  int64_t at[N];
#pragma unroll
  for (int u = 0; u < N; ++u) at[u] = i[u] < end ? i[u] : 0;
  auto tokens = [&](auto* ids) {
    int64_t id[N];
#pragma unroll
    for (int u = 0; u < N; ++u) id[u] = ids[at[u]];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      key[u] = inside(id[u], s.V);
      row[u] = (uint32_t)at[u];
    }
  };
  if (s.key) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      key[u] = s.key[at[u]];
      row[u] = s.row[at[u]];
    }
  } else if (s.id64) {
    tokens(static_cast<const int64_t*>(s.ids));
  } else {
    tokens(static_cast<const int32_t*>(s.ids));
  }
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs s, ZeroArgs z) {
  __shared__ uint32_t cnt[kMaxDigits];
  if ((int)blockIdx.x >= s.tiles) {
    zero_rows<kSortThreads>(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    return;
  }
  const int digits = 1 << s.bits;
  for (int d = threadIdx.x; d < digits; d += kSortThreads) cnt[d] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * s.per_tile;
  const int64_t i1 = i0 + s.per_tile < s.n ? i0 + s.per_tile : s.n;
  for (int64_t step = i0; step < i1; step += kSortStep) {
    int64_t i[kSortKeys];
    uint32_t key[kSortKeys], row[kSortKeys];
#pragma unroll
    for (int u = 0; u < kSortKeys; ++u) i[u] = step + kSortThreads * u + threadIdx.x;
    sort_keys(s, i, i1, key, row);
#pragma unroll
    for (int u = 0; u < kSortKeys; ++u)
      if (i[u] < i1) atomicAdd(&cnt[(key[u] >> s.shift) & (digits - 1)], 1u);  // counts: any order gives the same
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kSortThreads) s.counts[(int64_t)blockIdx.x * digits + d] = cnt[d];
}

// The rank of a key among the wave's keys with the same digit: those of the
// wave's earlier rounds (the counter), then the lanes below.  Lanes without a
// key take part with in = false.
__device__ __forceinline__ uint32_t wave_rank(uint32_t d, int bits, bool in, uint32_t* cnt) {
  const int lane = threadIdx.x & 63;
  uint64_t same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const uint64_t ones = __ballot((d >> b) & 1);
    same &= (d >> b) & 1 ? ones : ~ones;
  }
  const int first = in ? __ffsll((unsigned long long)same) - 1 : lane;
  uint32_t old = 0;
  if (in && lane == first) old = atomicAdd(&cnt[d], (uint32_t)__popcll(same));
  old = __shfl(old, first);
  return old + __popcll(same & (((uint64_t)1 << lane) - 1));
}

__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortArgs s, ZeroArgs z) {
  if ((int)blockIdx.x >= s.tiles) {
    zero_rows<kSortThreads>(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    return;
  }
  __shared__ uint32_t base[kMaxDigits];             // next place of each digit of this tile
  __shared__ uint32_t cnt[kSortWaves][kMaxDigits];  // keys of each digit in a wave, then their first place
  __shared__ uint32_t wsum[kSortWaves];
  const int digits = 1 << s.bits, tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  static_assert(kSortThreads >= kMaxDigits, "a thread per digit");
  // Digit d's keys of this tile start after all keys of smaller digits and
  // those of digit d in earlier tiles.
  uint32_t all = 0, before = 0;
  if (tid < digits) {
    for (int t0 = 0; t0 < s.tiles; t0 += kScan) {
      uint32_t c[kScan];
#pragma unroll
      for (int u = 0; u < kScan; ++u) c[u] = s.counts[(int64_t)(t0 + u < s.tiles ? t0 + u : t0) * digits + tid];
#pragma unroll
      for (int u = 0; u < kScan; ++u) {
        all += t0 + u < s.tiles ? c[u] : 0;
        before += t0 + u < (int)blockIdx.x ? c[u] : 0;
      }
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
    // a wave holds kSortKeys times 64 consecutive keys
    int64_t i[kSortKeys];
    uint32_t key[kSortKeys], row[kSortKeys], rank[kSortKeys];
#pragma unroll
    for (int u = 0; u < kSortKeys; ++u) i[u] = step + (w * kSortKeys + u) * 64 + lane;
    sort_keys(s, i, i1, key, row);
#pragma unroll
    for (int u = 0; u < kSortKeys; ++u)
      rank[u] = wave_rank((key[u] >> s.shift) & (digits - 1), s.bits, i[u] < i1, cnt[w]);
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
      if (i[u] < i1) {
        const uint32_t at = cnt[w][(key[u] >> s.shift) & (digits - 1)] + rank[u];
        s.key_out[at] = key[u];
        s.row_out[at] = row[u];
      }
    }
    __syncthreads();
  }
}

// Up to kSmallKeys keys there is a shorter way: the place of row i is the
// number of rows j with (token_j, j) < (token_i, i), counted over all rows,
// which a workgroup holds in LDS.  n^2 comparisons of two instructions beat the
// passes of the sort (four launches of 5 us) while launches and their gaps are
// what costs: 11 us for 8192 rows.  With the sums over 512 columns 8192 rows
// take 24 us this way, 9000 by the sort 30; 16384 rows 41 and 32.
constexpr int kSmallKeys = 8192, kRankThreads = 1024, kRankWaves = kRankThreads / 64;

// split: lanes that share a row's comparisons (1, 2 or 4); a workgroup ranks
// 64 / split rows, its waves and their lane groups taking blocks of 64 rows j
// in turn.  In a block before row i's own an equal token counts, in one after
// it doesn't: the comparison is against token_i + 1 or token_i.
__global__ __launch_bounds__(kRankThreads) void rank_kernel(SortArgs s, int split, ZeroArgs z) {
  __shared__ __attribute__((aligned(16))) uint32_t key[kSmallKeys];
  __shared__ uint32_t place[64];
  if ((int)blockIdx.x >= s.tiles) {
    zero_rows<kRankThreads>(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    return;
  }
  const int n = (int)s.n, blocks = (n + 63) / 64, tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  for (int i0 = tid; i0 < 64 * blocks; i0 += 4 * kRankThreads) {
    int64_t i[4];
    uint32_t k[4], row[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) i[u] = i0 + kRankThreads * u;
    sort_keys(s, i, n, k, row);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i[u] < 64 * blocks) key[i[u]] = i[u] < n ? k[u] : 0xffffffffu;
  }
  if (tid < 64) place[tid] = 0;
  __syncthreads();
  const int rows = 64 / split, li = lane & (rows - 1), i = blockIdx.x * rows + li;
  const uint32_t mine = key[i];  // i < 64 * blocks: rows divides 64
  uint32_t below = 0;
  for (int jb = w * split + lane / rows; jb < blocks; jb += kRankWaves * split) {
    const uint32_t* kj = key + 64 * jb;
    if (jb != i / 64) {
      const uint32_t bound = mine + (jb < i / 64);
#pragma unroll
      for (int j = 0; j < 64; j += 4) {
        const u32x4 k4 = *reinterpret_cast<const u32x4*>(kj + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) below += k4[e] < bound;
      }
    } else {
#pragma unroll 8
      for (int j = 0; j < 64; ++j) below += kj[j] < mine + (64 * jb + j < i);
    }
  }
  atomicAdd(&place[li], below);  // whole numbers: any order gives the same
  __syncthreads();
  if (tid < rows && i < n) {
    s.key_out[place[tid]] = mine;
    s.row_out[place[tid]] = (uint32_t)i;
  }
}

// ------------------------------------------------------------------ the sums
// A workgroup takes kGroup sorted places and kSlab columns, each of its waves
// kTile of the places; the workgroups of a group's columns come one after
// another, so that whole rows are on their way at a time (8192 rows of 4096
// columns, 3300 tokens, dy through the caches: 34 us, with the places first
// 41).  A fill of the table leaves its last 256 MB in the memory-side cache,
// from where they go to memory while the sums run: 30 us with dy past the
// caches, 42 through them (stores of the fill that go past that cache make the
// fill 38 us longer); 28 since the rows ahead are loaded without branches.
//
// A run of at most kTile rows belongs to the wave where it begins, which
// follows it past its places, so it is summed at once.  Of a longer run the
// waves that it crosses leave partial sums: in LDS, where the workgroup adds
// them in order, and of a run that also crosses workgroups those sums in `part`
// for the last kernel.  The last places before a wave's own, its own and those
// it may follow a run to fit its lanes, one each.
constexpr int kTile = 16, kGroup = 4 * kTile;
constexpr int kSlab = 64 * 8;
constexpr int kAhead = 4;  // rows on their way

struct SumArgs {
  int64_t n;
  const uint32_t* key;  // sorted tokens (outside the table: V, at the end)
  const uint32_t* row;
  float* part;          // [groups][2][H] of long runs: the one that enters the group, the one that leaves it
};

// The rows' addresses depend on nothing but the sorted list, so kAhead rows
// are read ahead, and where the sums add to the table so are its old rows, at
// the places where runs begin (read where a run ends, each costs a trip to
// memory).
template <typename T, bool PAST, bool ADD>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a, SumArgs s) {
  // A wave's partial sums: of a long run that enters it and of one that leaves it.
  __shared__ __attribute__((aligned(16))) float part[4][2][kSlab];
  __shared__ uint32_t enters[4], leaves[4];  // their tokens; V: there is none
  __shared__ uint32_t ends[4];               // whether the run that enters ends with the wave's places or before
  const uint32_t slabs = (a.H + kSlab - 1) / kSlab, group = blockIdx.x / slabs;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c0 = (blockIdx.x - group * slabs) * kSlab, c = c0 + 8 * lane;
  const bool in = c < a.H;
  const uint32_t V = (uint32_t)a.V;
  // lane kTile + u holds the wave's place u
  const int64_t at = (int64_t)group * kGroup + w * kTile - kTile + lane;
  const bool there = at >= 0 && at < s.n;
  const uint32_t my_key = there ? s.key[at] : V, my_row = there ? s.row[at] : 0;
  auto key_at = [&](int u) { return (uint32_t)__builtin_amdgcn_readlane(my_key, kTile + u); };
  auto row_at = [&](int u) { return (uint32_t)__builtin_amdgcn_readlane(my_row, kTile + u); };
  // the run with place u: [from, to), as far as the lanes reach
  auto run = [&](int u, int& from, int& to) {
    const uint64_t m = __ballot(my_key == key_at(u));
    from = __ffsll((unsigned long long)m) - 1 - kTile;
    to = 64 - __clzll(m) - kTile;
  };
  int first = 0, stop = 0;                // the places to sum
  bool enter = false, leave = false;      // the first run began before, the last goes on (long ones)
  uint32_t enter_key = V, leave_key = V;
  if (key_at(0) < V) {
    int from, to;
    stop = kTile;
    run(0, from, to);
    enter = from < 0;
    if (enter && to - from <= kTile) {  // short: the wave before sums it
      first = to;
      enter = false;
    }
    if (enter) {
      enter_key = key_at(0);
      if (lane == 0) ends[w] = to <= kTile;
    }
    if (key_at(kTile - 1) < V) {
      run(kTile - 1, from, to);
      if (to > kTile) {
        if (to - from <= kTile) stop = to;
        else leave = true;
      }
      if (leave && from >= 0) leave_key = key_at(kTile - 1);
    } else {
      stop = __popcll(__ballot(lane >= kTile && lane < 2 * kTile && my_key < V));
    }
  }
  if (lane == 0) {
    enters[w] = enter_key;
    leaves[w] = leave_key;
  }
  const Dropper drop(a.drop);
  Eight<T> x[kAhead];
  Eight<float> old[ADD ? kAhead : 1];
  auto begins = [&](int u) { return (u == first) | (key_at(u - 1) != key_at(u)); };
  const int width = a.H * (int)sizeof(T);
  auto load = [&](int u, int slot) {  // (nothing past the last place)
    const bool on = u < stop;
    const T* dy = static_cast<const T*>(a.dy) + (int64_t)row_at(u) * a.ldy;
    x[slot].template fetch<PAST>(row_buffer(dy, on ? width : 0), c);
    // The table's old row in a branch: as an empty buffer for rows that begin no
    // run these loads made long runs 5 to 12% slower, short ones 0.5 to 2% faster.
    if constexpr (ADD)
      if (on & begins(u))
        old[slot].template fetch<false>(row_buffer(a.dtable + (int64_t)key_at(u) * a.lddt, 4 * a.H), c);
    __builtin_amdgcn_sched_barrier(0);  // in this order: a wait for one is a wait for all before it
  };
#pragma unroll
  for (int v = 0; v < kAhead; ++v) load(first + v, v);
  float acc[8], base[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = base[e] = 0.f;
  for (int j = first; j < stop; j += kAhead) {
#pragma unroll
    for (int v = 0; v < kAhead; ++v) {
      const int u = j + v;
      const bool on = u < stop, last = u + 1 == stop;
      if (on) {
        float f[8];
        x[v].get(f);
        drop.apply((uint64_t)(a.drop.row0 + row_at(u)) * (a.H / 8) + c / 8, f);
        if (begins(u)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = f[e];
          if constexpr (ADD) old[v].get(base);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += f[e];
        }
      }
      load(u + kAhead, v);
      if (on & (last | begins(u + 1))) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = acc[e] * a.scale;
        if (enter | (last & leave)) {
          Eight<float>::store(&part[w][enter ? 0 : 1][8 * lane], o);
        } else {
          if constexpr (ADD) {
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += base[e];
          }
          if (in) Eight<float>::store(a.dtable + (int64_t)key_at(u) * a.lddt + c, o);
        }
        enter = false;
      }
    }
  }
  __syncthreads();
  // The waves' partial sums in order, two columns a thread.
  const int lc = 2 * threadIdx.x;
  if (c0 + lc >= a.H) return;
  float2 sum = {0.f, 0.f};
  uint32_t k = V;        // the open run
  bool before = false;   // it entered the group
  float* group_part = s.part + (int64_t)group * 2 * a.H + c0 + lc;
  for (int u = 0; u < 4; ++u) {
    if (enters[u] < V) {
      const float2 p = *reinterpret_cast<const float2*>(&part[u][0][lc]);
      if (k == V) before = true;
      k = enters[u];
      sum.x += p.x;
      sum.y += p.y;
      if (ends[u]) {
        float2* out = reinterpret_cast<float2*>(before ? group_part : a.dtable + (int64_t)k * a.lddt + c0 + lc);
        if (ADD && !before) {
          const float2 o = *out;
          sum.x += o.x;
          sum.y += o.y;
        }
        *out = sum;
        k = V;
        before = false;
        sum = {0.f, 0.f};
      }
    }
    if (leaves[u] < V) {
      k = leaves[u];
      sum = *reinterpret_cast<const float2*>(&part[u][1][lc]);
    }
  }
  if (k < V) *reinterpret_cast<float2*>(group_part + (before ? 0 : a.H)) = sum;
}

// The long runs across groups: the one that begins in this group and leaves
// it, if there is one, from the group's second partial sum and the following
// groups' first ones, in kJoinGroups rows of groups in turn and then in row
// order.  A row of groups takes kJoinRun partial sums in turn, kJoinRun of those
// sums in turn and then these, so that a token in all of 2^28 rows is the end of
// 64 + 64 + 256 additions and not of 2^20.  Most workgroups find none and end
// after one trip to memory.
constexpr int kJoinCols = 256, kJoinGroups = 4, kJoinRun = 64;
constexpr int kJoinThreads = kJoinCols / 4 * kJoinGroups;
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(EmbedArgs a, SumArgs s) {
  __shared__ __attribute__((aligned(16))) float red[kJoinGroups][kJoinCols];
  const int lane = threadIdx.x & 63;
  const int64_t t = blockIdx.x, i0 = t * kGroup;
  const uint32_t V = (uint32_t)a.V;
  static_assert(kGroup == 64, "a lane per place");
  if (i0 + kGroup >= s.n) return;
  const uint32_t mine = s.key[i0 + lane], after = s.key[i0 + kGroup];
  const uint32_t before = i0 > 0 ? s.key[i0 - 1] : V;
  const uint32_t k = (uint32_t)__builtin_amdgcn_readlane(mine, 63);
  if (k >= V || after != k) return;
  const int from = __ffsll((unsigned long long)__ballot(mine == k)) - 1;
  if (from == 0 && before == k) return;                                 // it began in an earlier group
  if (i0 + from + kTile >= s.n || s.key[i0 + from + kTile] != k) return;  // a short run
  int64_t end = t;  // the last group whose last place is the run's
  for (;;) {
    const int64_t p = (end + 1 + lane) * kGroup + kGroup - 1;
    const uint64_t no = ~__ballot(p < s.n && s.key[p] == k);
    if (no) {
      end += __ffsll((unsigned long long)no) - 1;
      break;
    }
    end += 64;
  }
  if ((end + 1) * kGroup < s.n && s.key[(end + 1) * kGroup] == k) ++end;  // it ends inside the next one
  const int lc = threadIdx.x % (kJoinCols / 4) * 4, grp = threadIdx.x / (kJoinCols / 4);
  const int c = blockIdx.y * kJoinCols + lc;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (c < a.H) {
    for (int64_t u = t + grp; u <= end;) {
      f32x4 mid = {0.f, 0.f, 0.f, 0.f};
      for (int i = 0; i < kJoinRun && u <= end; ++i) {
        const int64_t left = (end - u) / kJoinGroups + 1;
        const int n = left < kJoinRun ? (int)left : kJoinRun;
        f32x4 run = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int k = 0; k < n; ++k, u += kJoinGroups)
          run += *reinterpret_cast<const f32x4*>(s.part + (u * 2 + (u == t ? 1 : 0)) * a.H + c);
        mid += run;
      }
      sum += mid;
    }
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

// ------------------------------------------------------------------ few rows
// Up to kDirectRows rows need no sorted list: a workgroup takes row i and
// kSlab columns, finds the rows with i's token by comparing all tokens (each
// lane holds kDirectRows / 64 of them), ends if one comes before i, and else
// sums them, wave w those of rows 64 w and on, then the waves' sums in order.  The
// workgroups after those clear the rows that no token names (they find that
// out the same way), so the whole gradient is one launch: 256 rows of 512
// columns in 3.3 us (11 if all have one token), through the sorted list 15.  With
// four times the rows that gap closes, and one token in all of them costs 60
// us against 14.
constexpr int kDirectRows = 256, kDirectHeld = kDirectRows / 64, kDirectAhead = 8;

template <typename T>
__global__ __launch_bounds__(256) void embed_direct_kernel(EmbedArgs a, int sums) {
  __shared__ __attribute__((aligned(16))) float red[3][kSlab];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = (int)a.rows;
  const uint32_t V = (uint32_t)a.V;
  uint32_t held[kDirectHeld];  // tokens of rows 64 u + lane (no branch between the loads: one trip to memory)
  auto hold = [&](auto* ids) {
#pragma unroll
    for (int u = 0; u < kDirectHeld; ++u) {
      const int r = 64 * u + lane;
      const int64_t id = ids[r < n ? r : 0];
      held[u] = r < n ? inside(id, a.V) : V;
    }
  };
  if (a.id64) hold(static_cast<const int64_t*>(a.ids));
  else hold(static_cast<const int32_t*>(a.ids));
  if ((int)blockIdx.x >= sums) {
    const int64_t blocks = gridDim.x - sums;
    for (int64_t v = ((int64_t)blockIdx.x - sums) * 4 + w; v < a.V; v += blocks * 4) {
      bool named = false;
#pragma unroll
      for (int u = 0; u < kDirectHeld; ++u) named |= held[u] == (uint32_t)v;
      if (__ballot(named)) continue;
      for (int c = 4 * lane; c < a.H; c += 256)
        *reinterpret_cast<f32x4*>(a.dtable + v * a.lddt + c) = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    return;
  }
  const int slabs = (a.H + kSlab - 1) / kSlab, i = blockIdx.x / slabs;
  const int c = (blockIdx.x - i * slabs) * kSlab + 8 * lane;
  const bool in = c < a.H;
  uint32_t k = V;
#pragma unroll
  for (int u = 0; u < kDirectHeld; ++u)
    if (i / 64 == u) k = __builtin_amdgcn_readlane(held[u], i % 64);
  if (k >= V) return;
  uint64_t same[kDirectHeld];  // the rows with token k
#pragma unroll
  for (int u = 0; u < kDirectHeld; ++u) {
    same[u] = __ballot(held[u] == k);
    const int64_t before = (int64_t)i - 64 * u;  // rows of this word before i
    if (before > 0 && (before >= 64 ? same[u] : same[u] & (((uint64_t)1 << before) - 1))) return;
  }
  const Dropper drop(a.drop);
  uint64_t left = same[0];  // of the wave's rows
#pragma unroll
  for (int u = 1; u < kDirectHeld; ++u)
    if (w == u) left = same[u];
  const int mine = __popcll(left);
  Eight<T> x[kDirectAhead];
  int row[kDirectAhead];
  auto load = [&](int m, int slot) {
    if (m >= mine) return;
    row[slot] = 64 * w + __ffsll((unsigned long long)left) - 1;
    left &= left - 1;
    if (in) x[slot].load(static_cast<const T*>(a.dy) + (int64_t)row[slot] * a.ldy + c);
  };
#pragma unroll
  for (int v = 0; v < kDirectAhead; ++v) load(v, v);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  for (int j = 0; j < mine; j += kDirectAhead) {
#pragma unroll
    for (int v = 0; v < kDirectAhead; ++v) {
      if (j + v >= mine) break;
      float f[8];
      x[v].get(f);
      drop.apply((uint64_t)(a.drop.row0 + row[v]) * (a.H / 8) + c / 8, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += f[e];
      load(j + v + kDirectAhead, v);
    }
  }
  if (w > 0) Eight<float>::store(&red[w - 1][8 * lane], acc);
  __syncthreads();
  if (w > 0 || !in) return;
#pragma unroll
  for (int u = 0; u < 3; ++u) {
    float f[8];
    load8f(&red[u][8 * lane], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += f[e];
  }
  float* out = a.dtable + (int64_t)k * a.lddt + c;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] *= a.scale;
  if (a.accumulate) {
    float o[8];
    load8f(out, o);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += o[e];
  }
  Eight<float>::store(out, acc);
}

// ------------------------------------------------------------------ the plan
struct Plan {
  int64_t groups;  // of the sums
  int64_t keys, counts, part, bytes;  // byte offsets: four arrays of n words from 0, then these
};
Plan plan(int64_t rows, int H) {
  Plan p;
  p.groups = (rows + kGroup - 1) / kGroup;
  p.keys = (rows * 4 + 255) / 256 * 256;
  p.counts = 4 * p.keys;
  p.part = p.counts + (int64_t)kMaxSortTiles * kMaxDigits * 4;
  p.bytes = p.part + p.groups * 2 * (int64_t)H * 4;
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

template <typename T, bool PAST>
hipError_t backward(const EmbedArgs& a, hipStream_t stream) {
  if (a.rows <= kDirectRows) {
    const int64_t slabs = (a.H + kSlab - 1) / kSlab, most = 4 * (int64_t)device_cus();
    const int64_t zero = a.accumulate ? 0 : (a.V + 3) / 4 < most ? (a.V + 3) / 4 : most;
    hipLaunchKernelGGL(embed_direct_kernel<T>, dim3((unsigned)(a.rows * slabs + zero)), dim3(256), 0, stream, a,
                       (int)(a.rows * slabs));
    return hipGetLastError();
  }
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
  const int launches = a.rows <= kSmallKeys ? 1 : 2 * passes;  // of the sort: each clears its part of the table
  int part = 0;
  auto zeros = [&]() {
    ZeroArgs z{a.dtable, a.lddt, a.V * part / launches, a.V * (part + 1) / launches, a.H};
    ++part;
    if (a.accumulate) z.v0 = z.v1;
    return z;
  };
  // Workgroups of nt threads that clear z, four pieces a thread (524 MB under
  // the ranking of 8192 rows, with the sums: 129 us; 32 pieces and at most four
  // workgroups a compute unit: 137); zero_rows goes round where 2^20 are too few.
  auto zero_blocks = [&](const ZeroArgs& z, int64_t nt) {
    const int64_t b = ((z.v1 - z.v0) * (z.H / 4) + 4 * nt - 1) / (4 * nt), most = (int64_t)1 << 20;
    return (unsigned)(b < most ? b : most);
  };
  hipError_t e;
  if (a.rows <= kSmallKeys) {
    s.key_out = arr[0];
    s.row_out = arr[1];
    // as few rows a workgroup as it takes to occupy every compute unit
    const int split = a.rows <= 16 * (int64_t)device_cus() ? 4 : a.rows <= 32 * (int64_t)device_cus() ? 2 : 1;
    s.tiles = (int)((a.rows * split + 63) / 64);
    const ZeroArgs z = zeros();
    hipLaunchKernelGGL(rank_kernel, dim3((unsigned)s.tiles + zero_blocks(z, kRankThreads)), dim3(kRankThreads), 0,
                       stream, s, split, z);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    s.key = s.key_out;
    s.row = s.row_out;
  } else {
    for (int i = 0, at = 0; i < passes; ++i) {
      s.shift = at;
      s.bits = (bits - at + passes - i - 1) / (passes - i);
      at += s.bits;
      s.key_out = arr[2 * (i & 1)];
      s.row_out = arr[2 * (i & 1) + 1];
      ZeroArgs z = zeros();
      hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)s.tiles + zero_blocks(z, kSortThreads)), dim3(kSortThreads),
                         0, stream, s, z);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      z = zeros();
      hipLaunchKernelGGL(sort_scatter_kernel, dim3((unsigned)s.tiles + zero_blocks(z, kSortThreads)),
                         dim3(kSortThreads), 0, stream, s, z);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      s.key = s.key_out;
      s.row = s.row_out;
    }
  }
  SumArgs u{a.rows, s.key, s.row, reinterpret_cast<float*>(ws + p.part)};
  const dim3 grid((unsigned)(p.groups * ((a.H + kSlab - 1) / kSlab)));
  if (a.accumulate)
    hipLaunchKernelGGL((embed_sum_kernel<T, PAST, true>), grid, dim3(256), 0, stream, a, u);
  else
    hipLaunchKernelGGL((embed_sum_kernel<T, PAST, false>), grid, dim3(256), 0, stream, a, u);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(embed_join_kernel,
                     dim3((unsigned)p.groups, (unsigned)((a.H + kJoinCols - 1) / kJoinCols)), dim3(kJoinThreads), 0,
                     stream, a, u);
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
  if (stream_activation(a.rows, a.H, a.f32))
    return a.f32 ? backward<float, true>(a, stream) : backward<uint16_t, true>(a, stream);
  return a.f32 ? backward<float, false>(a, stream) : backward<uint16_t, false>(a, stream);
}

}  // namespace sppo
