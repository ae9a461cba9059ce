/*
 * libsppo -- sequence-chunked causal attention (forward + backward) with
 * per-chunk activation offload to pinned host memory, for one MI355X (gfx950).
 *
 * The method is the single-GPU slice of Sequence Pipeline Parallel Offloading
 * (SPPO, arXiv 2503.10377):
 *   - The sequence of length S is split into N subsequences ("chunks") with
 *     offsets c_0 = 0 < c_1 < ... < c_N = S (notation table: S, N, s_i).
 *   - A query of chunk i attends to the keys/values of chunks 0..i
 *     (Sec. 5.1, two-level activation management): every earlier chunk is
 *     fully visible, the diagonal block carries the causal mask.  Keys and
 *     values are the "skeletal" tensors and stay resident on the GPU.
 *   - The other saved activations of chunk i (here Q_i, O_i, LSE_i, and
 *     optionally a host copy of K_i/V_i) are offloaded to host memory while
 *     the next chunk computes, and must be back on the device before the
 *     backward of chunk i begins (Sec. 5.1, Sec. 5.2); page-locked host
 *     buffers give the full host-link bandwidth (Sec. 7, implementation).
 *   - The backward walks the chunks in reverse order and accumulates dK/dV.
 *
 * Layout (token-major BSHD, all tensors contiguous, device pointers unless
 * stated otherwise, every pointer 16-byte aligned):
 *   chunk-local  Q_i, O_i, dO_i, dQ_i : [B, s_i, Hq, D]   dtype of the problem
 *   chunk-local  LSE_i                : [B, Hq, s_i]      fp32, natural log
 *   full-length  K, V                 : [B, S, Hkv, D]    dtype of the problem
 *   full-length  dK, dV accumulators  : [B, S, Hkv, D]    fp32
 * Query head h reads KV head h / (Hq / Hkv).  With B = 1, chunk i of a full
 * [1, S, H, D] tensor is the contiguous slab starting at row c_i.
 *
 * Threading and streams: a context is used from one host thread at a time.
 * Every call is asynchronous with respect to the host on the stream it is
 * given (a hipStream_t passed as void*; NULL is the legacy null stream),
 * except sppo_copy_stats, sppo_sync and sppo_destroy, which block.  All
 * backward calls of one context must be issued on one stream (they share the
 * context's Delta workspace).
 *
 * Errors: every call returns an sppo_status.  Arguments are validated on the
 * host before anything is enqueued; a failed call enqueues nothing.  A HIP
 * error maps to SPPO_ERR_HIP; asynchronous device faults surface at the next
 * call that synchronises.  sppo_last_error() holds a message for the last
 * failure of that context.  Nothing aborts or throws across this ABI.
 */
#ifndef SPPO_H
#define SPPO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sppo_ctx sppo_ctx;

typedef enum {
  SPPO_OK = 0,
  SPPO_ERR_INVALID_ARG = 1, /* null/misaligned pointer, bad shape, bad index */
  SPPO_ERR_UNSUPPORTED = 2, /* valid but not implemented (e.g. head_dim)     */
  SPPO_ERR_ORDER = 3,       /* fwd not 0..N-1, or bwd not N-1..0           */
  SPPO_ERR_STATE = 4,       /* e.g. prefetch of a chunk never offloaded    */
  SPPO_ERR_OOM = 5,         /* device or pinned host allocation failed     */
  SPPO_ERR_HIP = 6          /* a HIP runtime call failed                   */
} sppo_status;

typedef enum { SPPO_F32 = 0, SPPO_BF16 = 1 } sppo_dtype;

/* Which saved activations of a chunk travel to host memory after its
 * forward (two-level activation management, Sec. 5.1).  In the first three
 * modes K/V stay resident on the device as the skeletal level. */
typedef enum {
  SPPO_OFFLOAD_NONE = 0,  /* nothing leaves the device                      */
  SPPO_OFFLOAD_QOL = 1,   /* Q_i, O_i, LSE_i offloaded and prefetched back  */
  SPPO_OFFLOAD_QKVOL = 2, /* as QOL, plus a host copy of K_i and V_i; the
                             resident K/V cache is not re-fetched           */
  SPPO_OFFLOAD_QKVOL_EVICT = 3
                          /* as QKVOL, but once the forward walk is over the
                             K/V cache rows of offloaded chunks count as
                             evicted (the caller may reuse that memory
                             after sppo_offload_wait): they come back with
                             sppo_prefetch_kv, and the backward of the last
                             chunk, the only one that runs before all of
                             them are back, does its dK/dV work one KV
                             chunk at a time, each piece waiting only for
                             its own rows, so the K/V copies stream in
                             under it                                      */
} sppo_offload;

/* The problem, in the paper's notation (B, S, N, s_i) plus the attention
 * shape (query heads, KV heads, head dim).  Copied by sppo_create, which
 * returns UNSUPPORTED when B or a head count exceeds 65535 or a
 * [B, S, max(Hq, Hkv), D] tensor would exceed 2^62 bytes. */
typedef struct {
  int64_t batch;                 /* B >= 1                                  */
  int64_t seq_len;               /* 1 <= S < 2^31 (kernels index keys in int) */
  int32_t n_chunks;              /* N, 1 <= N <= S                          */
  const int64_t* chunk_offsets;  /* host array of N+1 offsets, strictly
                                    increasing from 0 to S; NULL means N
                                    equal chunks (requires S % N == 0)      */
  int32_t n_q_heads;             /* Hq >= 1                                 */
  int32_t n_kv_heads;            /* Hkv >= 1, Hq % Hkv == 0                 */
  int32_t head_dim;              /* D in {64, 128}                          */
  sppo_dtype dtype;              /* element type of Q, K, V, O, dO, dQ      */
  float softmax_scale;           /* 0 means 1/sqrt(D)                       */
  sppo_offload offload;          /* offload set; NONE allocates no host mem */
  int32_t n_extra;               /* 0..16 further saved-activation planes
                                    that travel with Q/O/LSE (the rest of a
                                    full layer's saved tensors, Sec. 5.1:
                                    everything but K/V is offloadable)      */
  const size_t* extra_row_bytes; /* host array of n_extra row sizes (bytes
                                    per token, positive multiples of 4);
                                    plane k of chunk i is a
                                    chunk-local [B, s_i, extra_row_bytes[k]]
                                    byte array; NULL when n_extra == 0      */
} sppo_problem;

/* Device pointers of one chunk's saved activations, for offload/prefetch. */
typedef struct {
  void* q;      /* Q_i   [B, s_i, Hq, D]  chunk-local                        */
  void* o;      /* O_i   [B, s_i, Hq, D]  chunk-local                        */
  float* lse;   /* LSE_i [B, Hq, s_i]     chunk-local                        */
  void* k;      /* base of the full K cache [B, S, Hkv, D]; rows of chunk i  */
  void* v;      /* base of the full V cache [B, S, Hkv, D]; rows of chunk i  */
  void* const* extra; /* n_extra device pointers (planes of chunk i), or
                         NULL when the problem has no extra planes          */
  void* keep;   /* device buffer of sppo_keep_bytes(ctx, i) bytes, 16-byte
                   aligned, or NULL.  With sequence-aware offloading (rows_i
                   < s_i, see sppo_set_offload_rows) the rows [rows_i, s_i)
                   of Q_i, O_i, LSE_i and the extra planes stay on the
                   device.  With a keep buffer, sppo_offload_issue moves
                   them there (a copy kernel on its stream), so
                   the source buffers are dead as a whole after
                   sppo_offload_wait and can be reused (a device staging
                   ring), and sppo_prefetch moves them back into its
                   destination buffers (a copy kernel on its stream) -- pass the same
                   keep pointer to both.  Without one, they stay in the
                   source buffers, and the prefetch must target those same
                   buffers.  Ignored when rows_i == s_i.  The caller owns
                   the buffer and keeps it untouched from the offload to
                   the prefetch of chunk i.                                 */
} sppo_chunk_bufs;

typedef struct {
  uint64_t bytes_d2h;    /* bytes copied device->host since create/reset  */
  uint64_t bytes_h2d;    /* bytes copied host->device                     */
  double ms_d2h;         /* sum over chunks of event-timed D2H durations   */
  double ms_h2d;         /* sum over chunks of event-timed H2D durations   */
  int32_t n_d2h;         /* chunks offloaded                               */
  int32_t n_h2d;         /* chunks prefetched                              */
} sppo_copy_stats_t;

/* Kernels of one chunk, for per-kernel timing. */
typedef enum {
  SPPO_KERNEL_FWD = 0,       /* forward of a chunk                          */
  SPPO_KERNEL_BWD_PRE = 1,   /* Delta = rowsum(dO * O)                      */
  SPPO_KERNEL_BWD_DKDV = 2,  /* dK/dV accumulation over the chunk's queries */
  SPPO_KERNEL_BWD_DQ = 3,    /* dQ of the chunk                             */
  SPPO_KERNEL_COUNT = 4
} sppo_kernel;

typedef struct {
  double ms[SPPO_KERNEL_COUNT];         /* summed event-timed durations     */
  int32_t launches[SPPO_KERNEL_COUNT];  /* launches timed                   */
} sppo_kernel_times_t;

/* Create a context: validates the problem, copies the offsets, allocates
 * the Delta workspace (fp32 [B, Hq, max s_i]) on the current device and
 * per-chunk events, takes a reference on the device's two copy streams
 * (device->host and host->device, default priority, created by the first
 * context on the device and shared by all of its contexts, so the library
 * adds two streams to a process however many contexts it has), and --
 * unless offload is NONE -- allocates page-locked host slots for every
 * chunk's offload set.
 * *out is set only on success.  Errors: INVALID_ARG, UNSUPPORTED, OOM, HIP. */
sppo_status sppo_create(const sppo_problem* problem, sppo_ctx** out);

/* Synchronise the copy streams (which also waits for copies that other
 * contexts on the device have enqueued) and free everything the context
 * owns (the copy streams go when the last context on the device is
 * destroyed).  Safe on NULL. */
sppo_status sppo_destroy(sppo_ctx* ctx);

/* Forward of chunk i (Sec. 5.1): for rows r in [c_i, c_{i+1}) and every
 * query head, O_i[r] = softmax over keys j <= r (global positions) of
 * scale * Q_i[r].K[j], applied to V; LSE_i[r] = log sum_j exp(scale*Q.K).
 * Reads K/V rows [0, c_{i+1}).  Calls must come in order i = 0..N-1 (the
 * first call after create, after sppo_reset, or after bwd(0) must be
 * i = 0); otherwise ORDER and nothing is enqueued. */
sppo_status sppo_attn_fwd_chunk(sppo_ctx* ctx, int32_t i, const void* q_i,
                                const void* k, const void* v, void* o_i,
                                float* lse_i, void* stream);

/* Backward of chunk i in the reverse walk (Sec. 5.2): with Delta_r =
 * <dO_r, O_r>, P = exp(scale*Q.K - LSE), dS = P (dO.V - Delta):
 *   dQ_i = scale * dS K                         (written)
 *   dK[0, c_{i+1}) += scale * dS^T Q_i,  dV[0, c_{i+1}) += P^T dO_i
 * For i = N-1 (the first backward call) dK/dV rows [0, S) are overwritten,
 * so the accumulators need no zeroing; rows >= c_{i+1} are never touched.
 * Calls must come in order i = N-1..0 after fwd(N-1).  If chunk i was
 * offloaded, the stream first waits for the prefetch of chunk i, which must
 * have been issued (otherwise STATE).  With QKVOL_EVICT, bwd(N-1) requires
 * sppo_prefetch_kv of every offloaded chunk (otherwise STATE) and runs its
 * dK/dV kernel once per KV chunk j = N-1..0, each launch after chunk j's
 * K/V-ready event, then dQ. */
sppo_status sppo_attn_bwd_chunk(sppo_ctx* ctx, int32_t i, const void* q_i,
                                const void* k, const void* v, const void* o_i,
                                const float* lse_i, const void* do_i,
                                void* dq_i, float* dk_acc, float* dv_acc,
                                void* stream);

/* Offload chunk i's saved activations (the set chosen by problem.offload)
 * from the device pointers in *src to the context's pinned host slot i.
 * Records an event on `stream` (after the fwd of chunk i); the context's
 * D2H stream waits for it, copies, and records the chunk's offload-done
 * event.  The device sources must not be overwritten until that event --
 * see sppo_offload_wait.  Requires fwd(i) issued, offload != NONE. */
sppo_status sppo_offload_issue(sppo_ctx* ctx, int32_t i,
                               const sppo_chunk_bufs* src, void* stream);

/* Make `stream` wait until chunk i's offload copies have completed (its
 * device buffers may then be reused or overwritten).  Requires the offload
 * of chunk i to have been issued. */
sppo_status sppo_offload_wait(sppo_ctx* ctx, int32_t i, void* stream);

/* Prefetch chunk i's offloaded Q/O/LSE from host slot i into the device
 * pointers in *dst (K/V are never re-fetched: the cache is resident).  The
 * H2D stream waits for an event recorded now on `stream` (so dst may be
 * written after everything already enqueued there) and for chunk i's
 * offload-done event; the backward of chunk i then waits for the copy.
 * Requires the offload of chunk i to have been issued. */
sppo_status sppo_prefetch(sppo_ctx* ctx, int32_t i, const sppo_chunk_bufs* dst,
                          void* stream);

/* QKVOL_EVICT only: copy chunk i's K_i/V_i rows from host slot i back into
 * the device K/V cache (k, v: base pointers of the full [B, S, Hkv, D]
 * tensors) on the context's H2D stream, after everything already enqueued
 * on `stream` and after chunk i's offload has completed, and record chunk
 * i's K/V-ready event.  Allowed once the forward walk is over (in_bwd) and
 * before the backward of chunk N-1, which requires it for every offloaded
 * chunk and waits for chunk j's K/V-ready event right before the dK/dV work
 * on chunk j's key rows.  Errors: STATE (other mode, forward walk not over,
 * chunk not offloaded, already prefetched, backward already started),
 * INVALID_ARG. */
sppo_status sppo_prefetch_kv(sppo_ctx* ctx, int32_t i, void* k, void* v, void* stream);

/* Sequence-aware offloading (Sec. 5.2, adaptive offloading ratio alpha_i):
 * offload only the first `rows` rows (0 <= rows <= s_i) of chunk i's
 * offload set -- a row prefix of Q_i, O_i, LSE_i (and of K_i/V_i with
 * QKVOL*) -- and keep the rest resident; alpha_i = rows / s_i.  The default
 * is rows = s_i.  offload_issue, prefetch and prefetch_kv of chunk i then
 * move that prefix only (rows = 0 moves nothing but still orders the
 * streams).  Allowed only between walks (after create, reset or bwd(0)).
 * Errors: INVALID_ARG (index, rows out of range), STATE (mid-walk). */
sppo_status sppo_set_offload_rows(sppo_ctx* ctx, int32_t i, int64_t rows);

/* The offloaded row prefix of every chunk (n_chunks values). */
sppo_status sppo_get_offload_rows(const sppo_ctx* ctx, int64_t* out, int32_t capacity);

/* FLOPs-balanced partition (Sec. 3, computation imbalance of causal
 * attention; Sec. 5.2, FLOPs-based partition): chunk k of a causal
 * sequence covers about S^2 (2k+1) / (2N^2) of the S^2/2 visible (query,
 * key) pairs, so equal work per chunk needs c_k = S sqrt(k/N): long chunks
 * first, shorter ones later.  Writes N+1 offsets to out, each interior
 * offset rounded to a multiple of `align` and every chunk at least `align`
 * rows long.  Pure host function.  Errors: INVALID_ARG (S < N * align,
 * null out, N < 1, align < 1). */
sppo_status sppo_balanced_offsets(int64_t seq_len, int32_t n_chunks, int64_t align, int64_t* out);

/* Offload plan of sequence-aware offloading (Sec. 5.2): the copy of chunk i
 * should take no longer than the compute it overlaps, t_overlap_ms[i]
 * (normally the forward of chunk i+1), so with a device->host rate of
 * bw_GBps and bytes_per_row bytes of offload set per token row,
 *   rows_i = min(s_i, floor(bw * t_overlap_i / bytes_per_row)),
 * rounded down to a multiple of `align` when below s_i; the last chunk gets
 * rows = 0.  alpha_i = rows_i / s_i; alpha_i * A_i is then bounded by the
 * bytes the link moves in t_overlap_i.  Pure host function.  Errors:
 * INVALID_ARG. */
sppo_status sppo_plan_offload_rows(const int64_t* offsets, int32_t n_chunks, double bytes_per_row,
                                   double bw_GBps, const double* t_overlap_ms, int64_t align,
                                   int64_t* rows_out);

/* Bytes of chunk i's keep buffer (see sppo_chunk_bufs.keep) for its
 * current offload row count: 0 when the whole chunk is offloaded, or for an
 * invalid context or index. */
size_t sppo_keep_bytes(const sppo_ctx* ctx, int32_t i);

/* Finalize step of the reverse walk (optional): key j receives gradient
 * only from query rows r >= j, and the walk runs the backward of chunks
 * N-1, ..., 0 (Sec. 5.2), so once bwd(i) has been issued the dK/dV rows
 * [c_i, c_{i+1}) are final.  Writes those rows of every batch entry of
 * dk_out/dv_out ([B, S, Hkv, D] in the problem's dtype: fp32 accumulators
 * rounded to nearest even for bf16, copied for fp32) on `stream`, after
 * the backward enqueued there.  Rows outside the chunk are not touched.
 * Errors: STATE (bwd(i) not issued since the last fwd(0) or reset),
 * INVALID_ARG (null/misaligned pointers, dk_out == dv_out). */
sppo_status sppo_attn_finalize_chunk(sppo_ctx* ctx, int32_t i, const float* dk_acc, const float* dv_acc,
                                     void* dk_out, void* dv_out, void* stream);

/* Abandon the current forward/backward walk (e.g. after a forward-only run):
 * the next call must be fwd(0).  Blocks until the device's copy streams are
 * idle (copies of the abandoned walk may still read or write its device
 * buffers and host slots; the streams are shared, so this also waits for
 * copies other contexts have enqueued), then clears per-chunk offload state. */
sppo_status sppo_reset(sppo_ctx* ctx);

/* Block until the context's copy streams are idle. */
sppo_status sppo_sync(sppo_ctx* ctx);

/* Synchronise the copy streams and return cumulative copy statistics;
 * `reset_after` != 0 zeroes them afterwards. */
sppo_status sppo_copy_stats(sppo_ctx* ctx, sppo_copy_stats_t* out, int32_t reset_after);

/* Host-link rates of the context's own copy path, measured in isolation
 * (the "T_copy_iso" of the offload-hidden figure): allocates a device buffer
 * and a page-locked host buffer of `bytes` each, then times, on the
 * context's copy streams with events, one device->host copy, one
 * host->device copy, and both at once; frees the buffers and returns GB/s
 * (1e9 bytes per second).  Blocks the host.  Errors: INVALID_ARG (bytes <
 * 1 MiB), OOM, HIP. */
typedef struct {
  double d2h_GBps;     /* device->host alone                               */
  double h2d_GBps;     /* host->device alone                               */
  double duplex_GBps;  /* both directions at once, bytes of both / time    */
} sppo_link_rates_t;
sppo_status sppo_link_probe(sppo_ctx* ctx, size_t bytes, sppo_link_rates_t* out);

/* Enable (1) or disable (0) per-kernel timing: while enabled, every kernel
 * launch is bracketed by two events on the caller's stream.  Creates the
 * events on first use.  The backward of a small chunk is then launched kernel
 * by kernel too, where it otherwise does dK/dV and dQ in one launch: the same
 * results, but the times are those of the separate launches. */
sppo_status sppo_set_kernel_timing(sppo_ctx* ctx, int32_t enable);

/* Wait for the timed kernels and return the summed durations and launch
 * counts per kernel since the last reset; `reset_after` != 0 zeroes them. */
sppo_status sppo_kernel_times(sppo_ctx* ctx, sppo_kernel_times_t* out, int32_t reset_after);

/* The stream waits until chunk i's prefetch (sppo_prefetch) has landed, for
 * work other than the attention backward (which waits by itself) that
 * reads the prefetched tensors, e.g. the rest of a layer's backward.
 * STATE if chunk i's prefetch was not issued. */
sppo_status sppo_prefetch_wait(sppo_ctx* ctx, int32_t i, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the
 * backward of one chunk [c0, c1) as sppo_attn_bwd_chunk enqueues it (same
 * kernels, same results bit for bit), without a context and without any
 * allocation.  Its Delta / LSE workspace and the dK/dV kernel's tile
 * queues are a static device array of the library (8 MiB on every GPU the
 * library runs on, held until the process ends; the queues are cleared by
 * each call and left zero), so batch * n_q_heads * (c1 - c0) must not
 * exceed 2^20 (UNSUPPORTED otherwise, as for the size limits of
 * sppo_create).  Every call on one GPU shares that GPU's array: calls that
 * overlap on one GPU (several streams or threads) race, so the caller
 * orders them (e.g. one stream).  Arguments as in sppo_create and
 * sppo_attn_bwd_chunk: q_i, o_i, do_i, dq_i [B, c1 - c0, Hq, D] and lse_i
 * [B, Hq, c1 - c0] chunk-local; k, v [B, S, Hkv, D]; dk_acc, dv_acc fp32
 * [B, S, Hkv, D], rows [0, c1) overwritten (accumulate = 0) or added to
 * (accumulate = 1), rows >= c1 untouched.  No call-order checks (there is
 * no walk state).  Errors: INVALID_ARG, UNSUPPORTED, HIP, with the message
 * in sppo_last_error(NULL) on the calling thread. */
sppo_status sppo_attn_bwd_chunk_noalloc(int64_t batch, int64_t seq_len, int64_t c0, int64_t c1,
                                        int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                        sppo_dtype dtype, float softmax_scale, int32_t accumulate,
                                        const void* q_i, const void* k, const void* v, const void* o_i,
                                        const float* lse_i, const void* do_i, void* dq_i, float* dk_acc,
                                        float* dv_acc, void* stream);

/* Chunk offsets as stored by the context (n_chunks + 1 values). */
sppo_status sppo_get_offsets(const sppo_ctx* ctx, int64_t* out, int32_t capacity);

/* Message for the last failure of this context ("" if none); with
 * ctx == NULL, the message of the last failed sppo_create, context-free
 * attention call or training operator on this thread. */
const char* sppo_last_error(const sppo_ctx* ctx);

/* Static name of a status code. */
const char* sppo_status_string(sppo_status s);

/* ------------------------------------------------------------------------
 * Full-layer building blocks.  A transformer layer chunk (Sec. 5.1: the
 * subsequence's tensors of one layer -- LayerNorm, the QKV projection,
 * attention, the output projection and the MLP; Sec. 3.3: attention and the
 * GEMMs are the compute-bound operators) is composed from the attention
 * calls above and the calls below.  They need no context: each validates
 * its arguments on the host, enqueues on `stream` and returns a status
 * (INVALID_ARG, UNSUPPORTED or HIP); nothing is enqueued on failure.
 * Activations are bf16, statistics and parameter gradients fp32, every
 * pointer a device pointer, 16-byte aligned where it is bf16 data, every
 * leading dimension (ld*, in elements) a multiple of 8.
 * ---------------------------------------------------------------------- */

/* C[M, N] (op)= sum_k A(m, k) B(k, n), bf16 operands, fp32 accumulation.
 *   SPPO_GEMM_NT: A is [M, K] (row stride lda), B is [N, K] (ldb), so
 *                 C = A B^T; K % 64 == 0.  x W = x (W^T)^T with W^T
 *                 [out, in], and dY W^T with W [in, out].
 *   SPPO_GEMM_TN: A is stored [K, M], B stored [K, N], so C = A^T B;
 *                 M % 256 == 0, N % 256 == 0.  The weight gradient X^T dY.
 * Rows past M (NT) or K (TN) read as zero, only C[m < M][n < N] is
 * written.  Epilogues (aux: bf16 [M, N] with row stride ldaux):
 *   BF16      C = acc (bf16)
 *   ADD_BF16  C = acc + aux (bf16): the residual add
 *   GELU      aux = bf16(acc) (the pre-activation, kept for the backward),
 *             C = gelu(aux) with gelu(a) = a/2 (1 + tanh(sqrt(2/pi)(a +
 *             0.044715 a^3)))
 *   DGELU     C = acc * gelu'(aux) (bf16)
 *   ACC_F32   C += acc (fp32): gradients accumulated over chunks
 *   F32       C = acc (fp32)
 * N, ldc and ldaux must be multiples of 4 and aux 8-byte aligned (the
 * epilogues use 8- and 16-byte vector accesses): SPPO_ERR_INVALID_ARG
 * otherwise.  M * ldc and M * ldaux must stay below 2^31 elements (the
 * epilogue addresses C and aux by 32-bit element offsets):
 * SPPO_ERR_UNSUPPORTED otherwise. */
typedef enum { SPPO_GEMM_NT = 0, SPPO_GEMM_TN = 1 } sppo_gemm_layout;
typedef enum {
  SPPO_EPI_BF16 = 0,
  SPPO_EPI_ADD_BF16 = 1,
  SPPO_EPI_GELU = 2,
  SPPO_EPI_DGELU = 3,
  SPPO_EPI_ACC_F32 = 4,
  SPPO_EPI_F32 = 5
} sppo_epilogue;
sppo_status sppo_gemm_bf16(int32_t layout, int64_t M, int64_t N, int64_t K, const void* a, int64_t lda,
                           const void* b, int64_t ldb, void* c, int64_t ldc, int32_t epilogue, void* aux,
                           int64_t ldaux, void* stream);

/* LayerNorm of `rows` rows of H (H % 8 == 0, H <= 8192):
 * y = (x - mean) * rstd * gamma + beta, rstd = 1/sqrt(var + eps) with the
 * biased variance; mean and rstd (fp32 [rows]) are written for the
 * backward.  gamma, beta fp32 [H]. */
sppo_status sppo_layernorm_fwd(int64_t rows, int32_t H, const void* x, int64_t ldx, const float* gamma,
                               const float* beta, float eps, void* y, int64_t ldy, float* mean, float* rstd,
                               void* stream);

/* Backward of the LayerNorm above, with the residual branch folded in:
 *   dx = dres + rstd * (g - mean_j g - xhat * mean_j(g xhat)),
 *   g = dy * gamma, xhat = (x - mean) * rstd,
 * and dgamma (+)= sum_rows dy * xhat, dbeta (+)= sum_rows dy (fp32 [H];
 * accumulate != 0 adds, 0 overwrites; the sums run in a fixed order, so
 * results are reproducible bit for bit).  workspace: device fp32 scratch
 * of sppo_layernorm_bwd_workspace bytes. */
size_t sppo_layernorm_bwd_workspace(int64_t rows, int32_t H);
sppo_status sppo_layernorm_bwd(int64_t rows, int32_t H, const void* x, int64_t ldx, const float* gamma,
                               const float* mean, const float* rstd, const void* dy, int64_t lddy,
                               const void* dres, int64_t lddres, void* dx, int64_t lddx, float* dgamma,
                               float* dbeta, int32_t accumulate, float* workspace, size_t workspace_bytes,
                               void* stream);

/* y = gelu(x) (the tanh form above) over n bf16 values, n % 8 == 0. */
sppo_status sppo_gelu_bf16(const void* x, void* y, int64_t n, void* stream);

/* out [cols, rows] = in [rows, cols]^T, bf16, both contiguous. */
sppo_status sppo_transpose_bf16(const void* in, void* out, int64_t rows, int64_t cols, void* stream);

/* Row t < rows of out [rows, wq + 2 wkv] (bf16) = [dq[t] | dk[row0 + t] |
 * dv[row0 + t]]: the chunk's dQ (bf16 [rows, wq]) beside its rows of the
 * fp32 dK/dV accumulators ([.., wkv]) rounded to bf16 -- the gradient of
 * the fused QKV projection's output (B = 1). */
sppo_status sppo_pack_qkv_grad(int64_t rows, int32_t wq, int32_t wkv, const void* dq, const float* dk,
                               const float* dv, int64_t row0, void* out, void* stream);

/* ------------------------------------------------------------------------
 * Training operators beside the layer's: dropout, the norms, gate and
 * residual at a block's ends, and the token embedding.  Context-free like
 * the calls above (device pointers, validated on the host, nothing enqueued
 * on failure, the message in sppo_last_error(NULL) on the calling thread),
 * and free of any allocation or synchronisation, so they can be captured
 * into a graph.  `dtype` is the element type of every activation and of the
 * embedding table; parameters, statistics and parameter gradients are fp32.
 * Activations are row-major with a leading dimension in elements.  Widths
 * and leading dimensions are multiples of 8, activation, table and gradient
 * table pointers 16-byte aligned, the other pointers aligned to their type.
 * An output may be the same buffer as an input only where it says so.  A
 * workspace is the call's own until its work on the stream is done: calls
 * that may run at the same time (two streams, two graphs) need one each.
 * ---------------------------------------------------------------------- */

/* Dropout without a stored mask.  Whether an element is kept depends on
 * (seed, offset, its position in the whole sequence) alone, so the backward
 * and a recomputed forward draw the mask again, and the chunks of a sequence
 * draw the mask that the whole sequence would:
 *   t = row0 + r (r: row of the call), e = t * W + c (c < W: column, W the
 *   row's width), u = 16-bit half word e % 8 (low half of word 0 first) of
 *   Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as
 *   easy as 1, 2, 3", SC 2011) with counter words (e / 8 low, e / 8 high,
 *   offset low, offset high) and key (seed low, seed high);
 *   kept when u >= T, T = round(65536 p), and then scaled by
 *   65536 / (65536 - T), the inverse of the probability that is drawn.
 * A dropped element is zero whatever its value (NaN and infinities too).
 * Calls that need independent masks (other operators, other steps) take
 * other offsets.  offset_dev: NULL, or a device uint64 added to offset when
 * the kernel runs, so that a replayed graph draws new masks; it is to hold
 * the same value in a step's forward and backward. */
typedef struct {
  float p;                    /* 0 <= p < 1, T < 65536                      */
  uint64_t seed;
  uint64_t offset;
  const uint64_t* offset_dev;
  int64_t row0;               /* global index of the call's first row, >= 0 */
} sppo_drop;

/* y = res + keep * x (res NULL: y = keep * x) for rows x cols elements;
 * applied to a gradient it is the backward.  y may be x or res (with the
 * same leading dimension).  Errors: INVALID_ARG, UNSUPPORTED
 * ((row0 + rows) * cols >= 2^63), HIP. */
sppo_status sppo_dropout(sppo_dtype dtype, int64_t rows, int32_t cols, const void* x, int64_t ldx, const void* res,
                         int64_t ldres, const sppo_drop* drop, void* y, int64_t ldy, void* stream);

/* What joins a block's output b to the residual stream x, in one pass:
 *   n = N_post(b)                      (post NONE: n = b)
 *   h = residual_scale x + branch_scale keep (gate n)
 *   z = N_pre(h)                       (pre NONE: no z)
 * N is LayerNorm (LAYER: (v - mean) rstd gamma + beta, biased variance) or
 * RMSNorm (RMS: v rstd gamma + beta, rstd = 1/sqrt(mean(v^2) + eps)); beta
 * may be NULL (zero).  gate: fp32, one value per channel [H] (a parameter)
 * or per row [rows].  keep: the dropout above, W = H, or none.  H % 8 == 0,
 * H <= 8192, rows < 2^22 (UNSUPPORTED otherwise: the backward adds up to
 * rows / 256 rows of a column sum in turn, in fp32; a longer sequence goes in
 * calls of its parts, with drop's row0, and gradients that are added to).
 * Everything between the loads and the stores is fp32: z and its statistics
 * come from h before it is rounded. */
typedef enum { SPPO_NORM_NONE = 0, SPPO_NORM_LAYER = 1, SPPO_NORM_RMS = 2 } sppo_norm;
typedef enum { SPPO_GATE_NONE = 0, SPPO_GATE_CHANNEL = 1, SPPO_GATE_TOKEN = 2 } sppo_gate;
typedef struct {
  int32_t H;
  sppo_dtype dtype;
  sppo_norm post, pre;
  sppo_gate gate_kind;
  float eps;                /* where there is a norm: > 0, a normal number  */
  float residual_scale, branch_scale;  /* finite, |branch_scale| < 2^112    */
  const float* post_gamma;  /* [H], needed unless post is NONE              */
  const float* post_beta;   /* [H] or NULL                                  */
  const float* gate;        /* [H] or [rows], needed unless gate is NONE    */
  const float* pre_gamma;   /* [H], needed unless pre is NONE               */
  const float* pre_beta;    /* [H] or NULL                                  */
} sppo_block_norm;

/* Row statistics, fp32 [rows]: written by the forward, read by the
 * backward.  Each is needed where its norm is there (the means for LAYER
 * only) and ignored otherwise. */
typedef struct {
  float* post_mean;
  float* post_rstd;
  float* pre_mean;
  float* pre_rstd;
} sppo_block_norm_stats;

/* Parameter gradients, fp32 ([H]; gate as the gate).  NULL: not wanted.
 * One without its parameter is ignored. */
typedef struct {
  float* post_gamma;
  float* post_beta;
  float* gate;
  float* pre_gamma;
  float* pre_beta;
} sppo_block_norm_grads;

/* drop: NULL for none.  z: needed unless pre is NONE.  h may be x or b, and
 * z may be b (with the same leading dimension; h and z differ). */
sppo_status sppo_block_norm_fwd(const sppo_block_norm* bn, int64_t rows, const sppo_drop* drop, const void* x,
                                int64_t ldx, const void* b, int64_t ldb, void* h, int64_t ldh, void* z, int64_t ldz,
                                const sppo_block_norm_stats* stats, void* stream);

/* Backward: dz is z's gradient, dh the gradient that reaches h from
 * elsewhere (the residual stream; NULL: none, where there is a z).  With
 * D = dh + N_pre'(dz):
 *   dx = residual_scale D,  m = branch_scale keep D,  dgate = sum m n,
 *   db = N_post'(gate m),  and the norms' parameter gradients.
 * The [H] gradients are overwritten (accumulate = 0) or added to, their sums
 * over rows taken in a fixed order (the same bits every time); a gate
 * gradient per row is always written.  b is needed unless post is NONE and
 * no gate gradient is wanted, h where there is a z.  dx may be dh or dz, db
 * may be b, dz or h (with the same leading dimension; dx and db differ).
 * workspace: sppo_block_norm_bwd_workspace bytes (0 for an invalid bn; it
 * does not shrink as rows grow), 16-byte aligned. */
size_t sppo_block_norm_bwd_workspace(const sppo_block_norm* bn, int64_t rows);
sppo_status sppo_block_norm_bwd(const sppo_block_norm* bn, int64_t rows, const sppo_drop* drop, const void* b,
                                int64_t ldb, const void* h, int64_t ldh, const sppo_block_norm_stats* stats,
                                const void* dz, int64_t lddz, const void* dh, int64_t lddh, void* dx, int64_t lddx,
                                void* db, int64_t lddb, const sppo_block_norm_grads* grads, int32_t accumulate,
                                void* workspace, size_t workspace_bytes, void* stream);

/* y[r] = keep * (scale * table[ids[r]]), table [V, H] with row stride ldt,
 * |scale| < 2^112; ids [rows] of id_type.  An id outside [0, V) (padding,
 * another rank's part of a split vocabulary) gives a row of zeros whatever the
 * table holds (its row 0 may be read for it, and is not used).
 * drop: NULL for none (W = H).  rows <= 2^28, V < 2^31, H <= 2^20
 * and rows * H <= 2^38 (UNSUPPORTED otherwise; the gradient's too). */
typedef enum { SPPO_I32 = 0, SPPO_I64 = 1 } sppo_id_type;
sppo_status sppo_embedding_fwd(sppo_dtype dtype, sppo_id_type id_type, int64_t rows, int32_t H, int64_t V,
                               const void* ids, const void* table, int64_t ldt, float scale, const sppo_drop* drop,
                               void* y, int64_t ldy, void* stream);

/* Its gradient, by sorted tokens: dtable[v] (fp32 [V, H], row stride lddt)
 * = scale * sum over the rows r with ids[r] == v of keep * dy[r].
 * accumulate 0 overwrites all V rows (rows without a token become zero), 1
 * adds to the rows that have tokens and leaves the others as they are.  The
 * sums run in a fixed order, so results are the same bits every time.  Ids
 * outside [0, V) contribute nothing, and their rows of dy are not used.
 * workspace:
 * sppo_embedding_bwd_workspace bytes (0 for invalid sizes; it does not
 * shrink as rows grow), 16-byte aligned. */
size_t sppo_embedding_bwd_workspace(int64_t rows, int32_t H);
sppo_status sppo_embedding_bwd(sppo_dtype dtype, sppo_id_type id_type, int64_t rows, int32_t H, int64_t V,
                               const void* ids, const void* dy, int64_t lddy, float scale, const sppo_drop* drop,
                               float* dtable, int64_t lddt, int32_t accumulate, void* workspace,
                               size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * What closes a training step: positions in the attention, the loss, and the
 * update of the parameters.  Context-free calls under the rules of the ones
 * above: validated on the host, nothing enqueued on failure, no allocation,
 * no synchronisation, the message in sppo_last_error(NULL).
 * ---------------------------------------------------------------------- */

/* Rotary positions.  The first `rot` elements of a head are rot / 2 pairs:
 * (j, j + rot/2) in the HALF layout, (2j, 2j + 1) in INTERLEAVED.  A pair
 * (a, b) of a row at position t becomes
 *   amp (a cos w - b sin w,  b cos w + a sin w),  w = 2 pi t freqs[j] / 2^64
 * (inverse: -w, which with the same amp is the gradient); the elements from
 * rot on are copied.  freqs (device, [rot/2]) are fractions of a turn per
 * position in units of 2^-64, so that angles are exact modulo a turn: a
 * frequency that is off by 2^-63 turns puts position t off by |t| 2^-63.
 * positions: device [rows] of id_type, any values, or NULL for row0 + r.
 * The arithmetic is fp32, one rounding to the output's type. */
typedef enum { SPPO_ROTARY_HALF = 0, SPPO_ROTARY_INTERLEAVED = 1 } sppo_rotary_layout;
typedef struct {
  int32_t rot;              /* a multiple of 8, 8 <= rot                    */
  sppo_rotary_layout layout;
  const uint64_t* freqs;
  float amp;                /* finite                                       */
  sppo_id_type id_type;     /* of positions                                 */
  const void* positions;
  int64_t row0;
} sppo_rotary;

/* [rows, heads, head_dim] in memory: element (r, h, d) at r ld + h hs + d.
 * head_dim a multiple of 8, rot <= head_dim <= 1024; ld and hs multiples of 8,
 * with rows and heads apart from each other (hs >= head_dim and ld >= (heads
 * - 1) hs + head_dim, or ld >= head_dim and hs >= (rows - 1) ld + head_dim);
 * pointers 16-byte aligned.  y may be x with the same ld and hs; no other
 * overlap, also not between tensors of a call (INVALID_ARG where a y is another
 * tensor's x or y). */
typedef struct {
  sppo_dtype dtype;
  int32_t heads, head_dim;
  const void* x;
  int64_t ldx, hsx;
  void* y;
  int64_t ldy, hsy;
} sppo_rotary_tensor;

/* 1 to 4 tensors (queries and keys, or their gradients) of the same rows in
 * one launch.  tensors: host array.  rows 0: nothing is done. */
sppo_status sppo_rotary_apply(const sppo_rotary* spec, int64_t rows, int32_t inverse, int32_t n_tensors,
                              const sppo_rotary_tensor* tensors, void* stream);

/* The table of a rotary spec (a pure host function; freqs: host [rot/2], to be
 * copied to the device) and its amplitude.  With f_j = base^(-2j/rot), L =
 * original_len, s = factor:
 *   NONE    f_j, amp 1
 *   LINEAR  f_j / s, amp 1 (positions interpolated)
 *   NTK     f_j with base s^(rot / (rot - 2)), amp 1
 *   YARN    c f_j + (1 - c) f_j / s, c = clamp((L f_j / (2 pi) - beta_slow) /
 *           (beta_fast - beta_slow), 0, 1), amp 0.1 ln s + 1 (Peng, Quesnelle,
 *           Fan, Shippole, "YaRN", 2023)
 *   GIVEN   inv_freq[j] (host [rot/2], finite), amp 1
 * base > 1 (but for GIVEN), finite; s >= 1; YARN: L >= 1, beta_fast > beta_slow. */
typedef enum {
  SPPO_ROPE_NONE = 0,
  SPPO_ROPE_LINEAR = 1,
  SPPO_ROPE_NTK = 2,
  SPPO_ROPE_YARN = 3,
  SPPO_ROPE_GIVEN = 4
} sppo_rope_scaling;
typedef struct {
  sppo_rope_scaling kind;
  double base, factor;
  double original_len, beta_fast, beta_slow;
  const double* inv_freq;
} sppo_rope;
sppo_status sppo_rotary_freqs(int32_t rot, const sppo_rope* rope, uint64_t* freqs, float* amp);

/* Cross-entropy of rows of logits x over V classes, and its gradient:
 *   lse = log sum_c exp(x_c)
 *   loss = lse - (1 - e) x_t - (e / V) sum_c x_c + z lse^2
 *   dx_c = w ((1 + 2 z lse) exp(x_c - lse) - (1 - e) [c = t] - e / V)
 * with t the row's target, e = label_smoothing, z = z_loss, w = scale, times
 * *scale_dev (device fp32) where that is not NULL.  A row whose target is
 * outside [0, V) (padding) has loss, lse and gradient zero whatever its logits
 * hold.  Otherwise IEEE arithmetic holds: logits of -inf (masked classes) have
 * probability zero, a target at one has an infinite loss, and a row of nothing
 * but -inf has lse -inf and loss and gradient NaN.  With e > 0 a single -inf
 * makes the loss +inf.  Everything between logits and outputs is fp32. */
typedef struct {
  int64_t V;                /* 1 <= V < 2^31 (UNSUPPORTED above)            */
  sppo_dtype dtype;         /* of logits and dlogits                        */
  sppo_id_type id_type;     /* of targets                                   */
  float label_smoothing;    /* 0 <= e <= 1                                  */
  float z_loss;             /* finite, >= 0                                 */
  float scale;              /* finite                                       */
  const float* scale_dev;
} sppo_ce;

/* Loss and gradient in one call.  logits [rows, V] with row stride ld (V <=
 * ld, a multiple of 8, 16-byte aligned; V itself is any number), targets
 * [rows], loss and lse fp32 [rows] (lse may be NULL), dlogits as logits, or
 * NULL for the loss alone; it may be logits (with the same stride).  Columns
 * from V on are neither used nor written.  rows 0: nothing is done; rows <
 * 2^31.  workspace: sppo_cross_entropy_workspace bytes, 16-byte aligned: enough
 * for any call of up to that many rows (0 up to V = 32768, for no rows and for an
 * invalid ce).  Calls of V up to 131072 bf16 or 65536 fp32 logits and more than
 * 127 rows use none and take NULL, like those of V up to 32768. */
size_t sppo_cross_entropy_workspace(const sppo_ce* ce, int64_t rows);
sppo_status sppo_cross_entropy(const sppo_ce* ce, int64_t rows, const void* logits, int64_t ld, const void* targets,
                               float* loss, float* lse, void* dlogits, int64_t lddl, void* workspace,
                               size_t workspace_bytes, void* stream);

/* The gradient alone, from a kept lse; dloss: fp32 [rows], a factor beside the
 * scale, or NULL.  dlogits may be logits (with the same stride). */
sppo_status sppo_cross_entropy_bwd(const sppo_ce* ce, int64_t rows, const void* logits, int64_t ld,
                                   const void* targets, const float* lse, const float* dloss, void* dlogits,
                                   int64_t lddl, void* stream);

/* The parameters of an update, as one list for all its calls.  State:
 *   NONE  gradients only (for the norm)
 *   F32   m and v fp32 [n]
 *   E4M3  m and r = sqrt(v) in 8 bits: OCP e4m3 codes [n] under one power of two
 *         2^(b - 127) for 32 elements, b in m_scale, v_scale [ceil(n/32)] (all
 *         zeros is the state zero).  b is the least, from 1 on, with which the
 *         block's largest magnitude is at most 448 2^(b - 127).
 * A bf16 parameter has its fp32 master (which is what is updated, the parameter
 * its rounding); an fp32 parameter has none.  Pointers are aligned to their
 * element, with E4M3 to 16 bytes (the scales to 1).  n 0: skipped. */
typedef enum { SPPO_STATE_NONE = 0, SPPO_STATE_F32 = 1, SPPO_STATE_E4M3 = 2 } sppo_opt_state;
typedef struct {
  int64_t n;
  void* param;
  const void* grad;
  float* master;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  sppo_dtype param_dtype, grad_dtype;
  float lr_scale;           /* a factor of the learning rate, finite        */
  float weight_decay;       /* finite                                       */
} sppo_opt_tensor;

/* A list is made on the host (pure host functions), its table copied by the
 * caller to device memory (16-byte aligned) whose address it writes into
 * `table`; list and table live as long as their calls run.  INVALID_ARG where
 * a buffer that is written overlaps another of the list (a tensor listed twice;
 * gradients may be shared).  At most 2^20 tensors and 2^24 - 1 tiles of 2048
 * elements (UNSUPPORTED above). */
typedef struct {
  const void* table;
  int64_t tiles;
  int32_t n_tensors;
  sppo_opt_state state;
} sppo_opt_list;
size_t sppo_opt_list_bytes(int32_t n_tensors, const sppo_opt_tensor* tensors);
sppo_status sppo_opt_list_make(int32_t n_tensors, const sppo_opt_tensor* tensors, sppo_opt_state state,
                               void* host_table, size_t bytes, sppo_opt_list* list);

/* out (device fp32 [2]) = { norm, min(1, max_norm / norm) }, norm = the root of
 * the sum of the squares of all gradients, summed in fp64 in a fixed order (the
 * same bits every time).  max_norm > 0; infinity: the factor is 1.  A norm of
 * infinity (or past fp32's range) or NaN has the factor 0.  steps: NULL, or a device int64 that is
 * increased by one unless the norm is infinite or NaN.  workspace:
 * sppo_grad_norm_workspace bytes, 16-byte aligned. */
size_t sppo_grad_norm_workspace(const sppo_opt_list* list);
sppo_status sppo_grad_norm(const sppo_opt_list* list, float max_norm, float* out, int64_t* steps, void* workspace,
                           size_t workspace_bytes, void* stream);

/* One AdamW update of the list's parameters:
 *   g' = f g;  m = beta1 m + (1 - beta1) g';  v = beta2 v + (1 - beta2) g'^2
 *   p -= lr (m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay p)
 * t = step, plus *step_dev where that is not NULL (t >= 1, checked only where
 * the host knows it; below 1 on the device counts as 1); f = norm[1] and nothing
 * at all is changed where norm[0] is infinite or NaN (norm: a grad_norm's out,
 * NULL: f = 1); lr is multiplied by *lr_dev (device fp32) where that is not
 * NULL, and by the tensor's lr_scale.  Arithmetic is fp32.
 * With E4M3 the new m and r are rounded to the neighbour above with the
 * probability of what lies between (in 2^-16), and a positive r never to zero:
 * element e of a tensor whose blocks of 32 start at the list's block B takes
 * word e % 4 of Philox4x32-10 (as the dropout's) with counter (8 B + e / 4 low,
 * high, t low, high) and key seed, its low half for m, its high half for r.
 * Values that are infinite or NaN are kept as NaN, a v below 2^-126 as zero.
 * Squares past fp32's range: with F32 v is infinite from then on, and the
 * parameter only decays (is NaN from the next step on with beta2 0); with E4M3 m
 * and r are finite where they and g' were, kept to 240 2^120 (3.19e38). */
typedef struct {
  double lr, beta1, beta2, eps;  /* lr finite; 0 <= beta < 1; eps > 0, a
                                    normal fp32 number                      */
  int64_t step;
  const int64_t* step_dev;
  const float* norm;
  const float* lr_dev;
  uint64_t seed;
} sppo_adamw;
sppo_status sppo_adamw_step(const sppo_opt_list* list, const sppo_adamw* adamw, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SPPO_H */
