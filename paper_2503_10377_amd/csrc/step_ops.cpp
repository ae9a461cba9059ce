// C ABI of the operators that close a training step (rotary positions,
// cross-entropy, gradient norm, AdamW): each call validates its arguments on
// the host, enqueues its kernels on the given stream and returns a status,
// with the message in sppo_last_error(NULL).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <string>
#include <vector>

#include "sppo.h"
#include "sppo_kernels.h"

namespace {

sppo_status fail(sppo_status st, const char* msg) {
  try {
    sppo::set_thread_error(msg);
  } catch (...) {  // no memory for the message: the status says enough
  }
  return st;
}

sppo_status launched(hipError_t e) {
  if (e == hipSuccess) return SPPO_OK;
  return fail(SPPO_ERR_HIP, hipGetErrorString(e));
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool dtype_ok(int dtype) { return dtype == SPPO_F32 || dtype == SPPO_BF16; }
bool id_type_ok(int t) { return t == SPPO_I32 || t == SPPO_I64; }
constexpr int64_t kFar = (int64_t)1 << 61;  // past any element offset

// ------------------------------------------------------------------- rotary
// Whether (r, h) -> r ld + h hs keeps rows and heads of D elements apart, with
// offsets that fit.
bool strides_ok(int64_t rows, int heads, int D, int64_t ld, int64_t hs) {
  if (ld <= 0 || hs <= 0 || ld % 8 || hs % 8 || ld > kFar / rows || hs > kFar / heads) return false;
  return (hs >= D && ld >= (int64_t)(heads - 1) * hs + D) || (ld >= D && hs >= (rows - 1) * ld + D);
}

// ---------------------------------------------------------------------- loss
sppo_status check_ce(const sppo_ce* ce) {
  if (!ce || !dtype_ok(ce->dtype) || !id_type_ok(ce->id_type))
    return fail(SPPO_ERR_INVALID_ARG, "cross entropy: no description, or unknown dtype or id type");
  if (ce->V < 1) return fail(SPPO_ERR_INVALID_ARG, "cross entropy: V < 1");
  if (ce->V > INT32_MAX) return fail(SPPO_ERR_UNSUPPORTED, "cross entropy: V above 2^31 - 1");
  if (!(ce->label_smoothing >= 0.f) || !(ce->label_smoothing <= 1.f) || !(ce->z_loss >= 0.f) ||
      !std::isfinite(ce->z_loss) || !std::isfinite(ce->scale))
    return fail(SPPO_ERR_INVALID_ARG,
                "cross entropy: label_smoothing outside [0, 1], z_loss negative or not finite, or scale not finite");
  if (!aligned(ce->scale_dev, 4)) return fail(SPPO_ERR_INVALID_ARG, "cross entropy: scale_dev is misaligned");
  return SPPO_OK;
}

sppo_status ce_args(const sppo_ce* ce, int64_t rows, const void* logits, int64_t ld, const void* targets,
                    void* dlogits, int64_t lddl, sppo::CeArgs* a) {
  const sppo_status st = check_ce(ce);
  if (st != SPPO_OK) return st;
  if (rows < 0) return fail(SPPO_ERR_INVALID_ARG, "cross entropy: rows < 0");
  if (rows > INT32_MAX) return fail(SPPO_ERR_UNSUPPORTED, "cross entropy: rows above 2^31 - 1");
  const auto mat_ok = [&](const void* p, int64_t l) {
    return p && aligned(p, 16) && l >= ce->V && l % 8 == 0 && (rows == 0 || l <= kFar / rows);
  };
  if (!mat_ok(logits, ld) || (dlogits && !mat_ok(dlogits, lddl)))
    return fail(SPPO_ERR_INVALID_ARG, "cross entropy: null or misaligned pointer, or bad leading dimension");
  if (dlogits == logits && ld != lddl)
    return fail(SPPO_ERR_INVALID_ARG, "cross entropy: dlogits over logits with another leading dimension");
  if (!targets || !aligned(targets, ce->id_type == SPPO_I64 ? 8 : 4))
    return fail(SPPO_ERR_INVALID_ARG, "cross entropy: null or misaligned targets");
  *a = sppo::CeArgs{};
  a->rows = rows;
  a->V = ce->V;
  a->x = logits; a->ldx = ld;
  a->targets = targets; a->id64 = ce->id_type == SPPO_I64;
  a->smooth = ce->label_smoothing; a->z = ce->z_loss;
  a->scale = ce->scale; a->scale_dev = ce->scale_dev;
  a->dx = dlogits; a->lddx = lddl;
  a->f32 = ce->dtype == SPPO_F32;
  return SPPO_OK;
}

// ---------------------------------------------------------------- parameters
constexpr int32_t kMaxTensors = 1 << 20;
constexpr int64_t kMaxTiles = ((int64_t)1 << 24) - 1;  // a workgroup of 256 each: 32 bits of threads

int64_t tiles_of(int64_t n) { return n / sppo::kOptTile + (n % sppo::kOptTile != 0); }
int64_t blocks_of(int64_t n) { return n / 32 + (n % 32 != 0); }

// Tiles of a list; negative where its sizes are not allowed.
int64_t count_tiles(int32_t n_tensors, const sppo_opt_tensor* t) {
  if (n_tensors < 1 || n_tensors > kMaxTensors || !t) return -1;
  int64_t tiles = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    if (t[i].n < 0) return -1;
    tiles += tiles_of(t[i].n);
    if (tiles > kMaxTiles) return -1;
  }
  return tiles;
}

size_t list_bytes(int32_t n_tensors, int64_t tiles) {
  return (size_t)n_tensors * sizeof(sppo::OptDesc) + (size_t)tiles * sizeof(sppo::OptTile);
}

sppo_status check_list(const sppo_opt_list* l) {
  if (!l || !l->table || !aligned(l->table, 16) || l->n_tensors < 1 || l->n_tensors > kMaxTensors || l->tiles < 0 ||
      l->tiles > kMaxTiles || l->state < SPPO_STATE_NONE || l->state > SPPO_STATE_E4M3)
    return fail(SPPO_ERR_INVALID_ARG, "optimizer: no list, or one without its table in device memory");
  return SPPO_OK;
}

sppo::OptTable table_of(const sppo_opt_list* l) {
  const auto* d = static_cast<const sppo::OptDesc*>(l->table);
  return {d, reinterpret_cast<const sppo::OptTile*>(d + l->n_tensors), l->tiles};
}

struct Span {
  uintptr_t lo, hi;
  bool written;
};

// A tensor's pointers for the list's state, as spans of memory.
sppo_status check_tensor(const sppo_opt_tensor& t, int state, std::vector<Span>& spans) {
  if (!dtype_ok(t.grad_dtype)) return fail(SPPO_ERR_INVALID_ARG, "optimizer: unknown gradient dtype");
  const uintptr_t wide = state == SPPO_STATE_E4M3 ? 16 : 0;
  const int64_t gs = t.grad_dtype == SPPO_BF16 ? 2 : 4, ps = t.param_dtype == SPPO_BF16 ? 2 : 4;
  const auto add = [&](const void* p, int64_t count, int64_t size, uintptr_t align, bool written) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    if (!p || !aligned(p, align)) return false;
    spans.push_back({lo, lo + (uintptr_t)(count * size), written});
    return true;
  };
  const auto at = [&](int64_t size) { return wide ? wide : (uintptr_t)size; };
  if (!add(t.grad, t.n, gs, at(gs), false))
    return fail(SPPO_ERR_INVALID_ARG, "optimizer: a null or misaligned gradient");
  if (state == SPPO_STATE_NONE) return SPPO_OK;
  if (!dtype_ok(t.param_dtype)) return fail(SPPO_ERR_INVALID_ARG, "optimizer: unknown parameter dtype");
  if (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay))
    return fail(SPPO_ERR_INVALID_ARG, "optimizer: lr_scale or weight_decay not finite");
  if ((t.param_dtype == SPPO_BF16) != (t.master != nullptr))
    return fail(SPPO_ERR_INVALID_ARG, "optimizer: a bf16 parameter has a master, an fp32 one has none");
  const bool small = state == SPPO_STATE_E4M3;
  const int64_t ss = small ? 1 : 4;
  if (!add(t.param, t.n, ps, at(ps), true) || (t.master && !add(t.master, t.n, 4, at(4), true)) ||
      !add(t.m, t.n, ss, at(ss), true) || !add(t.v, t.n, ss, at(ss), true) ||
      (small && (!add(t.m_scale, blocks_of(t.n), 1, 1, true) || !add(t.v_scale, blocks_of(t.n), 1, 1, true))))
    return fail(SPPO_ERR_INVALID_ARG, "optimizer: a null or misaligned parameter, master or state");
  return SPPO_OK;
}

// No written span meets another.  By their starts: a span that begins before an
// earlier one ends meets it, and one of the two must not be written.
bool apart(std::vector<Span>& spans) {
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
  uintptr_t end = 0, written_end = 0;
  for (const Span& s : spans) {
    if (s.lo < written_end || (s.written && s.lo < end)) return false;
    end = std::max(end, s.hi);
    if (s.written) written_end = std::max(written_end, s.hi);
  }
  return true;
}

}  // namespace

extern "C" {

sppo_status sppo_rotary_apply(const sppo_rotary* spec, int64_t rows, int32_t inverse, int32_t n_tensors,
                              const sppo_rotary_tensor* tensors, void* stream) {
  if (!spec || (spec->layout != SPPO_ROTARY_HALF && spec->layout != SPPO_ROTARY_INTERLEAVED) ||
      !id_type_ok(spec->id_type))
    return fail(SPPO_ERR_INVALID_ARG, "rotary: no description, or unknown layout or id type");
  if (spec->rot < 8 || spec->rot % 8 || !std::isfinite(spec->amp))
    return fail(SPPO_ERR_INVALID_ARG, "rotary: rot is not a positive multiple of 8, or amp is not finite");
  if (!spec->freqs || !aligned(spec->freqs, 8) || !aligned(spec->positions, spec->id_type == SPPO_I64 ? 8 : 4))
    return fail(SPPO_ERR_INVALID_ARG, "rotary: null or misaligned freqs, or misaligned positions");
  if (rows < 0 || (inverse != 0 && inverse != 1)) return fail(SPPO_ERR_INVALID_ARG, "rotary: bad rows or inverse");
  if (n_tensors < 1 || n_tensors > sppo::kRotaryMaxTensors || !tensors)
    return fail(SPPO_ERR_INVALID_ARG, "rotary: 1 to 4 tensors");
  sppo::RotaryArgs a{};
  for (int i = 0; i < n_tensors; ++i) {
    const sppo_rotary_tensor& t = tensors[i];
    if (!dtype_ok(t.dtype) || t.heads < 1 || t.head_dim < 8 || t.head_dim % 8 || t.head_dim < spec->rot)
      return fail(SPPO_ERR_INVALID_ARG,
                  "rotary: unknown dtype, no heads, or head_dim not a multiple of 8 of at least rot");
    if (t.head_dim > sppo::kRotaryMaxDim || t.heads > 65535)
      return fail(SPPO_ERR_UNSUPPORTED, "rotary: head_dim above 1024 or more than 65535 heads");
    if (!t.x || !t.y || !aligned(t.x, 16) || !aligned(t.y, 16))
      return fail(SPPO_ERR_INVALID_ARG, "rotary: null or misaligned pointer");
    const int64_t r = rows ? rows : 1;
    if (!strides_ok(r, t.heads, t.head_dim, t.ldx, t.hsx) || !strides_ok(r, t.heads, t.head_dim, t.ldy, t.hsy) ||
        (t.x == t.y && (t.ldx != t.ldy || t.hsx != t.hsy)))
      return fail(SPPO_ERR_INVALID_ARG, "rotary: bad strides");
    sppo::RotaryTensor& o = a.t[i];
    o.x = t.x; o.ldx = t.ldx; o.hsx = t.hsx;
    o.y = t.y; o.ldy = t.ldy; o.hsy = t.hsy;
    o.heads = t.heads; o.D = t.head_dim;
    o.f32 = t.dtype == SPPO_F32;
    for (int k = 0; k < i; ++k)
      if (t.y == tensors[k].y || t.y == tensors[k].x || t.x == tensors[k].y)
        return fail(SPPO_ERR_INVALID_ARG, "rotary: a tensor is written and used by another one of the call");
  }
  if (rows == 0) return SPPO_OK;
  a.rows = rows;
  a.rot = spec->rot; a.half = spec->layout == SPPO_ROTARY_HALF; a.n = n_tensors;
  a.freqs = spec->freqs;
  a.amp = spec->amp; a.sign = inverse ? -1.f : 1.f;
  a.pos = spec->positions; a.id64 = spec->id_type == SPPO_I64;
  a.row0 = spec->row0;
  return launched(sppo::launch_rotary(a, static_cast<hipStream_t>(stream)));
}

sppo_status sppo_rotary_freqs(int32_t rot, const sppo_rope* r, uint64_t* freqs, float* amp) {
  if (rot < 8 || rot % 8 || rot > sppo::kRotaryMaxDim || !r || !freqs || !amp)
    return fail(SPPO_ERR_INVALID_ARG, "rotary: rot is not a multiple of 8 in [8, 1024], or a null pointer");
  const int kind = r->kind;
  if (kind < SPPO_ROPE_NONE || kind > SPPO_ROPE_GIVEN) return fail(SPPO_ERR_INVALID_ARG, "rotary: unknown scaling");
  const bool given = kind == SPPO_ROPE_GIVEN, yarn = kind == SPPO_ROPE_YARN;
  if (given ? !r->inv_freq : !(r->base > 1.0 && std::isfinite(r->base)))
    return fail(SPPO_ERR_INVALID_ARG, "rotary: base is not above 1, or no inv_freq");
  if (!given && kind != SPPO_ROPE_NONE && !(r->factor >= 1.0 && std::isfinite(r->factor)))
    return fail(SPPO_ERR_INVALID_ARG, "rotary: factor is below 1 or not finite");
  if (yarn && !(r->original_len >= 1.0 && std::isfinite(r->original_len) && std::isfinite(r->beta_fast) &&
                std::isfinite(r->beta_slow) && r->beta_fast > r->beta_slow))
    return fail(SPPO_ERR_INVALID_ARG, "rotary: original_len below 1, or beta_fast not above beta_slow");
  const long double two_pi = 6.283185307179586476925286766559005768L, s = r->factor;
  for (int j = 0; given && j < rot / 2; ++j)
    if (!std::isfinite(r->inv_freq[j])) return fail(SPPO_ERR_INVALID_ARG, "rotary: a frequency is not finite");
  const long double base =
      kind == SPPO_ROPE_NTK ? r->base * std::pow(s, (long double)rot / (rot - 2)) : (long double)r->base;
  for (int j = 0; j < rot / 2; ++j) {
    long double f = given ? (long double)r->inv_freq[j] : std::pow(base, -2.0L * j / rot);
    if (kind == SPPO_ROPE_LINEAR) f /= s;
    if (yarn) {
      long double c = (r->original_len * f / two_pi - r->beta_slow) / ((long double)r->beta_fast - r->beta_slow);
      c = std::min(1.0L, std::max(0.0L, c));
      f = c * f + (1.0L - c) * f / s;
    }
    long double turns = f / two_pi;
    turns -= std::floor(turns);
    const long double u = std::nearbyint(std::ldexp(turns, 64));
    freqs[j] = u >= 18446744073709551616.0L ? 0 : (uint64_t)u;
  }
  *amp = yarn ? (float)(0.1L * std::log(s) + 1.0L) : 1.f;
  return SPPO_OK;
}

size_t sppo_cross_entropy_workspace(const sppo_ce* ce, int64_t rows) {
  if (check_ce(ce) != SPPO_OK || rows < 0 || rows > INT32_MAX) return 0;
  return sppo::cross_entropy_workspace(rows, ce->V, ce->dtype == SPPO_F32);
}

sppo_status sppo_cross_entropy(const sppo_ce* ce, int64_t rows, const void* logits, int64_t ld, const void* targets,
                               float* loss, float* lse, void* dlogits, int64_t lddl, void* workspace,
                               size_t workspace_bytes, void* stream) {
  sppo::CeArgs a;
  const sppo_status st = ce_args(ce, rows, logits, ld, targets, dlogits, lddl, &a);
  if (st != SPPO_OK) return st;
  if (!loss || !aligned(loss, 4) || !aligned(lse, 4))
    return fail(SPPO_ERR_INVALID_ARG, "cross entropy: null or misaligned loss, or misaligned lse");
  const size_t need = sppo::cross_entropy_uses(rows, ce->V, a.f32);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
    return fail(SPPO_ERR_INVALID_ARG, "cross entropy: workspace null, misaligned or too small");
  if (rows == 0) return SPPO_OK;
  a.loss = loss;
  a.lse = lse;
  a.workspace = workspace;
  return launched(sppo::launch_cross_entropy(a, static_cast<hipStream_t>(stream)));
}

sppo_status sppo_cross_entropy_bwd(const sppo_ce* ce, int64_t rows, const void* logits, int64_t ld,
                                   const void* targets, const float* lse, const float* dloss, void* dlogits,
                                   int64_t lddl, void* stream) {
  sppo::CeArgs a;
  const sppo_status st = ce_args(ce, rows, logits, ld, targets, dlogits, lddl, &a);
  if (st != SPPO_OK) return st;
  if (!dlogits || !lse || !aligned(lse, 4) || !aligned(dloss, 4))
    return fail(SPPO_ERR_INVALID_ARG, "cross entropy: no dlogits, null or misaligned lse, or misaligned dloss");
  if (rows == 0) return SPPO_OK;
  a.lse_in = lse;
  a.dloss = dloss;
  return launched(sppo::launch_cross_entropy_bwd(a, static_cast<hipStream_t>(stream)));
}

size_t sppo_opt_list_bytes(int32_t n_tensors, const sppo_opt_tensor* tensors) {
  const int64_t tiles = count_tiles(n_tensors, tensors);
  return tiles < 0 ? 0 : list_bytes(n_tensors, tiles);
}

sppo_status sppo_opt_list_make(int32_t n_tensors, const sppo_opt_tensor* tensors, sppo_opt_state state,
                               void* host_table, size_t bytes, sppo_opt_list* list) {
  if (!tensors || !host_table || !list || n_tensors < 1 || (int)state < SPPO_STATE_NONE || (int)state > SPPO_STATE_E4M3)
    return fail(SPPO_ERR_INVALID_ARG, "optimizer: a null pointer, no tensors or an unknown state");
  for (int32_t i = 0; i < n_tensors; ++i)
    if (tensors[i].n < 0) return fail(SPPO_ERR_INVALID_ARG, "optimizer: a tensor of negative size");
  const int64_t tiles = count_tiles(n_tensors, tensors);
  if (tiles < 0) return fail(SPPO_ERR_UNSUPPORTED, "optimizer: more than 2^20 tensors or 2^24 - 1 tiles");
  if (!aligned(host_table, 8) || bytes < list_bytes(n_tensors, tiles))
    return fail(SPPO_ERR_INVALID_ARG, "optimizer: the table is misaligned or too small");
  try {
    std::vector<Span> spans;
    for (int32_t i = 0; i < n_tensors; ++i) {
      if (tensors[i].n == 0) continue;
      const sppo_status st = check_tensor(tensors[i], state, spans);
      if (st != SPPO_OK) return st;
    }
    if (!apart(spans)) return fail(SPPO_ERR_INVALID_ARG, "optimizer: a buffer that is written overlaps another");
  } catch (...) {
    return fail(SPPO_ERR_OOM, "optimizer: no host memory to check the list");
  }
  auto* desc = static_cast<sppo::OptDesc*>(host_table);
  auto* tile = reinterpret_cast<sppo::OptTile*>(desc + n_tensors);
  int64_t block0 = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const sppo_opt_tensor& t = tensors[i];
    sppo::OptDesc d{};
    d.grad = t.grad;
    d.n = t.n;
    d.block0 = block0;
    d.flags = t.grad_dtype == SPPO_BF16 ? sppo::kOptGradBf16 : 0;
    if (state != SPPO_STATE_NONE) {
      d.param = t.param; d.master = t.master;
      d.m = t.m; d.v = t.v;
      d.m_scale = t.m_scale; d.v_scale = t.v_scale;
      d.lr_scale = t.lr_scale; d.weight_decay = t.weight_decay;
      if (t.param_dtype == SPPO_BF16) d.flags |= sppo::kOptParamBf16;
    }
    std::memcpy(desc + i, &d, sizeof d);
    block0 += blocks_of(t.n);
    const int64_t n_tiles = tiles_of(t.n);
    for (int64_t k = 0; k < n_tiles; ++k) *tile++ = {(uint32_t)i, (uint32_t)k};
  }
  *list = {nullptr, tiles, n_tensors, state};
  return SPPO_OK;
}

size_t sppo_grad_norm_workspace(const sppo_opt_list* list) {
  return list && list->tiles >= 0 && list->tiles <= kMaxTiles ? sppo::kNormBlocks * sizeof(double) : 0;
}

sppo_status sppo_grad_norm(const sppo_opt_list* list, float max_norm, float* out, int64_t* steps, void* workspace,
                           size_t workspace_bytes, void* stream) {
  const sppo_status st = check_list(list);
  if (st != SPPO_OK) return st;
  if (!(max_norm > 0.f)) return fail(SPPO_ERR_INVALID_ARG, "gradient norm: max_norm must be positive");
  if (!out || !aligned(out, 4) || !aligned(steps, 8))
    return fail(SPPO_ERR_INVALID_ARG, "gradient norm: null or misaligned out, or misaligned steps");
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < sppo_grad_norm_workspace(list))
    return fail(SPPO_ERR_INVALID_ARG, "gradient norm: workspace null, misaligned or too small");
  return launched(sppo::launch_grad_norm(table_of(list), max_norm, out, steps, static_cast<double*>(workspace),
                                         static_cast<hipStream_t>(stream)));
}

sppo_status sppo_adamw_step(const sppo_opt_list* list, const sppo_adamw* w, void* stream) {
  const sppo_status st = check_list(list);
  if (st != SPPO_OK) return st;
  if (list->state == SPPO_STATE_NONE) return fail(SPPO_ERR_INVALID_ARG, "adamw: the list has gradients only");
  if (!w || !std::isfinite((float)w->lr) || !(w->beta1 >= 0.0) || !(w->beta1 < 1.0) || !(w->beta2 >= 0.0) ||
      !(w->beta2 < 1.0) || !((float)w->eps > 0.f) || !std::isnormal((float)w->eps))
    return fail(SPPO_ERR_INVALID_ARG,
                "adamw: lr not finite, eps not positive and a normal number, or a beta outside [0, 1)");
  if (!w->step_dev && w->step < 1) return fail(SPPO_ERR_INVALID_ARG, "adamw: step below 1");
  if (!aligned(w->step_dev, 8) || !aligned(w->norm, 4) || !aligned(w->lr_dev, 4))
    return fail(SPPO_ERR_INVALID_ARG, "adamw: a misaligned pointer");
  if (list->tiles == 0) return SPPO_OK;
  sppo::AdamArgs a{};
  a.beta1 = w->beta1; a.beta2 = w->beta2;
  a.lr = (float)w->lr; a.eps = (float)w->eps;
  a.step = w->step;
  a.step_dev = w->step_dev;
  if (!w->step_dev) {
    a.im = (float)(1.0 / (1.0 - sppo::beta_power(w->beta1, w->step)));
    a.ir = (float)(1.0 / std::sqrt(1.0 - sppo::beta_power(w->beta2, w->step)));
  }
  a.norm = w->norm;
  a.lr_dev = w->lr_dev;
  a.seed = w->seed;
  return launched(sppo::launch_adamw(table_of(list), list->state, a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
