// C ABI of the training operators (dropout, block norms, embedding): each
// call validates its arguments on the host, enqueues its kernels on the given
// stream and returns a status, with the message in sppo_last_error(NULL).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <string>

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

// A row-major activation of `width` columns.
bool act_ok(const void* p, int64_t ld, int64_t width) { return p && aligned(p, 16) && ld >= width && ld % 8 == 0; }

// A scale that the kernels multiply with the dropout's (at most 65536): finite
// after that, so that it leaves a dropped element zero.
bool scale_ok(float scale) { return std::isfinite(scale * 65536.f); }

// The dropout of rows x width elements; NULL: none.
sppo_status drop_args(const sppo_drop* d, int64_t rows, int64_t width, sppo::DropArgs* out) {
  *out = sppo::DropArgs{};
  if (!d) return SPPO_OK;
  if (!(d->p >= 0.f) || !(d->p < 1.f)) return fail(SPPO_ERR_INVALID_ARG, "dropout: p must be in [0, 1)");
  const uint32_t t = (uint32_t)std::floor((double)d->p * 65536.0 + 0.5);
  if (t > 65535) return fail(SPPO_ERR_INVALID_ARG, "dropout: p rounds to 1 in units of 1/65536");
  if (d->row0 < 0) return fail(SPPO_ERR_INVALID_ARG, "dropout: row0 is negative");
  if (!aligned(d->offset_dev, 8)) return fail(SPPO_ERR_INVALID_ARG, "dropout: offset_dev is not 8-byte aligned");
  if (rows > INT64_MAX - d->row0 || d->row0 + rows > INT64_MAX / width)
    return fail(SPPO_ERR_UNSUPPORTED, "dropout: element index past 2^63");
  out->seed = d->seed;
  out->offset = d->offset;
  out->offset_dev = t ? d->offset_dev : nullptr;
  out->threshold = t;
  out->scale = 65536.f / (65536.f - (float)t);
  out->row0 = d->row0;
  return SPPO_OK;
}

// What a block norm's description says about itself.
sppo_status check_norm(const sppo_block_norm* bn, int64_t rows) {
  if (!bn || !dtype_ok(bn->dtype)) return fail(SPPO_ERR_INVALID_ARG, "block norm: no description, or unknown dtype");
  if (rows <= 0 || bn->H <= 0 || bn->H % 8 || bn->H > sppo::kBnMaxH)
    return fail(SPPO_ERR_INVALID_ARG, "block norm: rows < 1, or H not a multiple of 8 in [8, 8192]");
  const int post = bn->post, pre = bn->pre, gate = bn->gate_kind;
  if (post < SPPO_NORM_NONE || post > SPPO_NORM_RMS || pre < SPPO_NORM_NONE || pre > SPPO_NORM_RMS ||
      gate < SPPO_GATE_NONE || gate > SPPO_GATE_TOKEN)
    return fail(SPPO_ERR_INVALID_ARG, "block norm: unknown norm or gate");
  if ((post != SPPO_NORM_NONE || pre != SPPO_NORM_NONE) && !(bn->eps > 0.f && std::isnormal(bn->eps)))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: eps must be positive and a normal number");
  if (!std::isfinite(bn->residual_scale) || !scale_ok(bn->branch_scale))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: a scale is not finite, or branch_scale 2^112 and above");
  if ((post != SPPO_NORM_NONE && !bn->post_gamma) || (pre != SPPO_NORM_NONE && !bn->pre_gamma) ||
      (gate != SPPO_GATE_NONE && !bn->gate))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: a norm without gamma, or no gate values");
  if (!aligned(bn->post_gamma, 4) || !aligned(bn->post_beta, 4) || !aligned(bn->gate, 4) ||
      !aligned(bn->pre_gamma, 4) || !aligned(bn->pre_beta, 4))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: a misaligned parameter");
  // A thread of the backward adds up to rows / 256 rows (rows of one team's width
  // and more) of a column in turn: 16384 here, 2^-10 of the terms' magnitudes.
  if (rows >= (int64_t)1 << 22) return fail(SPPO_ERR_UNSUPPORTED, "block norm: more than 2^22 - 1 rows");
  return SPPO_OK;
}

sppo_status check_stats(const sppo_block_norm* bn, const sppo_block_norm_stats* s) {
  if (bn->post == SPPO_NORM_NONE && bn->pre == SPPO_NORM_NONE) return SPPO_OK;
  if (!s || (bn->post != SPPO_NORM_NONE && !s->post_rstd) || (bn->post == SPPO_NORM_LAYER && !s->post_mean) ||
      (bn->pre != SPPO_NORM_NONE && !s->pre_rstd) || (bn->pre == SPPO_NORM_LAYER && !s->pre_mean))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: a norm without its statistics");
  if (!aligned(s->post_mean, 4) || !aligned(s->post_rstd, 4) || !aligned(s->pre_mean, 4) || !aligned(s->pre_rstd, 4))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: misaligned statistics");
  return SPPO_OK;
}

sppo::BlockNormArgs norm_args(const sppo_block_norm* bn, int64_t rows, const sppo_block_norm_stats* s) {
  sppo::BlockNormArgs a{};
  a.rows = rows;
  a.H = bn->H;
  a.post = bn->post; a.pre = bn->pre; a.gate_kind = bn->gate_kind;
  a.eps = bn->eps; a.alpha = bn->residual_scale; a.bscale = bn->branch_scale;
  a.post_gamma = bn->post_gamma; a.post_beta = bn->post_beta;
  a.gate = bn->gate;
  a.pre_gamma = bn->pre_gamma; a.pre_beta = bn->pre_beta;
  if (s) {
    a.post_mean = s->post_mean; a.post_rstd = s->post_rstd;
    a.pre_mean = s->pre_mean; a.pre_rstd = s->pre_rstd;
  }
  a.f32 = bn->dtype == SPPO_F32;
  return a;
}

// Sizes that the embedding's kernels take: rows and V index as 32-bit numbers,
// and the columns' workgroups fit a grid's second dimension.
sppo_status check_embedding(int dtype, int id_type, int64_t rows, int32_t H, int64_t V, const void* ids, float scale) {
  if (!dtype_ok(dtype) || (id_type != SPPO_I32 && id_type != SPPO_I64))
    return fail(SPPO_ERR_INVALID_ARG, "embedding: unknown dtype or id type");
  if (rows <= 0 || V <= 0 || H <= 0 || H % 8) return fail(SPPO_ERR_INVALID_ARG, "embedding: bad rows, V or H");
  if (!ids || !aligned(ids, id_type == SPPO_I64 ? 8 : 4))
    return fail(SPPO_ERR_INVALID_ARG, "embedding: null or misaligned ids");
  if (!scale_ok(scale)) return fail(SPPO_ERR_INVALID_ARG, "embedding: the scale is not finite, or 2^112 and above");
  if (rows > sppo::kMaxEmbedRows || V > INT32_MAX || H > sppo::kMaxEmbedH || rows > sppo::kMaxEmbedElems / H)
    return fail(SPPO_ERR_UNSUPPORTED, "embedding: rows above 2^28, V above 2^31 - 1, H above 2^20 or rows * H above 2^38");
  return SPPO_OK;
}

}  // namespace

extern "C" {

sppo_status sppo_dropout(sppo_dtype dtype, int64_t rows, int32_t cols, const void* x, int64_t ldx, const void* res,
                         int64_t ldres, const sppo_drop* drop, void* y, int64_t ldy, void* stream) {
  if (!dtype_ok(dtype)) return fail(SPPO_ERR_INVALID_ARG, "dropout: unknown dtype");
  if (rows <= 0 || cols <= 0 || cols % 8) return fail(SPPO_ERR_INVALID_ARG, "dropout: bad rows or cols");
  if (!drop) return fail(SPPO_ERR_INVALID_ARG, "dropout: no sppo_drop");
  if (!act_ok(x, ldx, cols) || !act_ok(y, ldy, cols) || (res && !act_ok(res, ldres, cols)))
    return fail(SPPO_ERR_INVALID_ARG, "dropout: null or misaligned pointer, or bad leading dimension");
  sppo::DropoutArgs a{};
  const sppo_status st = drop_args(drop, rows, cols, &a.drop);
  if (st != SPPO_OK) return st;
  a.rows = rows;
  a.cols = cols;
  a.x = x; a.ldx = ldx;
  a.res = res; a.ldres = ldres;
  a.y = y; a.ldy = ldy;
  a.f32 = dtype == SPPO_F32;
  return launched(sppo::launch_dropout(a, static_cast<hipStream_t>(stream)));
}

sppo_status sppo_block_norm_fwd(const sppo_block_norm* bn, int64_t rows, const sppo_drop* drop, const void* x,
                                int64_t ldx, const void* b, int64_t ldb, void* h, int64_t ldh, void* z, int64_t ldz,
                                const sppo_block_norm_stats* stats, void* stream) {
  sppo_status st = check_norm(bn, rows);
  if (st == SPPO_OK) st = check_stats(bn, stats);
  if (st != SPPO_OK) return st;
  const bool pre = bn->pre != SPPO_NORM_NONE;
  if (!act_ok(x, ldx, bn->H) || !act_ok(b, ldb, bn->H) || !act_ok(h, ldh, bn->H) || (pre && !act_ok(z, ldz, bn->H)))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: null or misaligned pointer, or bad leading dimension");
  if (pre && h == z) return fail(SPPO_ERR_INVALID_ARG, "block norm: h and z are the same buffer");
  sppo::BlockNormArgs a = norm_args(bn, rows, stats);
  if ((st = drop_args(drop, rows, bn->H, &a.drop)) != SPPO_OK) return st;
  a.x = x; a.ldx = ldx;
  a.b = b; a.ldb = ldb;
  a.h = h; a.ldh = ldh;
  a.z = z; a.ldz = ldz;
  return launched(sppo::launch_block_norm_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t sppo_block_norm_bwd_workspace(const sppo_block_norm* bn, int64_t rows) {
  if (check_norm(bn, rows) != SPPO_OK) return 0;
  return sppo::block_norm_bwd_workspace(norm_args(bn, rows, nullptr));
}

sppo_status sppo_block_norm_bwd(const sppo_block_norm* bn, int64_t rows, const sppo_drop* drop, const void* b,
                                int64_t ldb, const void* h, int64_t ldh, const sppo_block_norm_stats* stats,
                                const void* dz, int64_t lddz, const void* dh, int64_t lddh, void* dx, int64_t lddx,
                                void* db, int64_t lddb, const sppo_block_norm_grads* grads, int32_t accumulate,
                                void* workspace, size_t workspace_bytes, void* stream) {
  sppo_status st = check_norm(bn, rows);
  if (st == SPPO_OK) st = check_stats(bn, stats);
  if (st != SPPO_OK) return st;
  sppo::BlockNormArgs a = norm_args(bn, rows, stats);
  if ((st = drop_args(drop, rows, bn->H, &a.drop)) != SPPO_OK) return st;
  if (accumulate != 0 && accumulate != 1) return fail(SPPO_ERR_INVALID_ARG, "block norm: accumulate must be 0 or 1");
  const bool post = bn->post != SPPO_NORM_NONE, pre = bn->pre != SPPO_NORM_NONE, gate = bn->gate_kind != SPPO_GATE_NONE;
  if (grads) {
    if (!aligned(grads->post_gamma, 4) || !aligned(grads->post_beta, 4) || !aligned(grads->gate, 4) ||
        !aligned(grads->pre_gamma, 4) || !aligned(grads->pre_beta, 4))
      return fail(SPPO_ERR_INVALID_ARG, "block norm: a misaligned gradient");
    a.d_post_gamma = post ? grads->post_gamma : nullptr;
    a.d_post_beta = post && bn->post_beta ? grads->post_beta : nullptr;
    a.d_gate = gate ? grads->gate : nullptr;
    a.d_pre_gamma = pre ? grads->pre_gamma : nullptr;
    a.d_pre_beta = pre && bn->pre_beta ? grads->pre_beta : nullptr;
  }
  const bool need_b = post || a.d_gate;
  if ((need_b && !act_ok(b, ldb, bn->H)) || (pre && (!act_ok(h, ldh, bn->H) || !act_ok(dz, lddz, bn->H))) ||
      (!pre && !dh) || (dh && !act_ok(dh, lddh, bn->H)) || !act_ok(dx, lddx, bn->H) || !act_ok(db, lddb, bn->H))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: null or misaligned pointer, or bad leading dimension");
  if (dx == db) return fail(SPPO_ERR_INVALID_ARG, "block norm: dx and db are the same buffer");
  const size_t need = sppo_block_norm_bwd_workspace(bn, rows);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
    return fail(SPPO_ERR_INVALID_ARG, "block norm: workspace null, misaligned or too small");
  a.b = need_b ? b : nullptr; a.ldb = ldb;
  a.h = const_cast<void*>(h); a.ldh = ldh;
  a.dz = dz; a.lddz = lddz;
  a.dh = dh; a.lddh = lddh;
  a.dx = dx; a.lddx = lddx;
  a.db = db; a.lddb = lddb;
  a.accumulate = accumulate;
  a.part = static_cast<float*>(workspace);
  return launched(sppo::launch_block_norm_bwd(a, static_cast<hipStream_t>(stream)));
}

sppo_status sppo_embedding_fwd(sppo_dtype dtype, sppo_id_type id_type, int64_t rows, int32_t H, int64_t V,
                               const void* ids, const void* table, int64_t ldt, float scale, const sppo_drop* drop,
                               void* y, int64_t ldy, void* stream) {
  sppo_status st = check_embedding(dtype, id_type, rows, H, V, ids, scale);
  if (st != SPPO_OK) return st;
  if (!act_ok(table, ldt, H) || !act_ok(y, ldy, H))
    return fail(SPPO_ERR_INVALID_ARG, "embedding: null or misaligned pointer, or bad leading dimension");
  sppo::EmbedArgs a{};
  if ((st = drop_args(drop, rows, H, &a.drop)) != SPPO_OK) return st;
  a.rows = rows; a.H = H; a.V = V;
  a.ids = ids; a.id64 = id_type == SPPO_I64;
  a.table = table; a.ldt = ldt;
  a.y = y; a.ldy = ldy;
  a.scale = scale;
  a.f32 = dtype == SPPO_F32;
  return launched(sppo::launch_embedding_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t sppo_embedding_bwd_workspace(int64_t rows, int32_t H) {
  if (rows <= 0 || rows > sppo::kMaxEmbedRows || H <= 0 || H % 8 || H > sppo::kMaxEmbedH || rows > sppo::kMaxEmbedElems / H)
    return 0;
  return sppo::embedding_workspace(rows, H);
}

sppo_status sppo_embedding_bwd(sppo_dtype dtype, sppo_id_type id_type, int64_t rows, int32_t H, int64_t V,
                               const void* ids, const void* dy, int64_t lddy, float scale, const sppo_drop* drop,
                               float* dtable, int64_t lddt, int32_t accumulate, void* workspace,
                               size_t workspace_bytes, void* stream) {
  sppo_status st = check_embedding(dtype, id_type, rows, H, V, ids, scale);
  if (st != SPPO_OK) return st;
  if (!act_ok(dy, lddy, H) || !act_ok(dtable, lddt, H))
    return fail(SPPO_ERR_INVALID_ARG, "embedding: null or misaligned pointer, or bad leading dimension");
  if (accumulate != 0 && accumulate != 1) return fail(SPPO_ERR_INVALID_ARG, "embedding: accumulate must be 0 or 1");
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < sppo_embedding_bwd_workspace(rows, H))
    return fail(SPPO_ERR_INVALID_ARG, "embedding: workspace null, misaligned or too small");
  sppo::EmbedArgs a{};
  if ((st = drop_args(drop, rows, H, &a.drop)) != SPPO_OK) return st;
  a.rows = rows; a.H = H; a.V = V;
  a.ids = ids; a.id64 = id_type == SPPO_I64;
  a.dy = dy; a.ldy = lddy;
  a.scale = scale;
  a.dtable = dtable; a.lddt = lddt;
  a.accumulate = accumulate;
  a.workspace = workspace;
  a.f32 = dtype == SPPO_F32;
  return launched(sppo::launch_embedding_bwd(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
