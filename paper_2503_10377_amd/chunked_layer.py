"""One full transformer layer over a chunked sequence, composed of libsppo
calls: the forward walks the chunks 0..N-1, the backward N-1..0 (Sec. 5.1-5.2
of SPPO), batch 1.

The layer (pre-LayerNorm GPT block, MLP width 4H, no projection biases):
    u = LN1(x); q, k, v = u W_qkv; O = causal attention; h = x + O W_o
    z = LN2(h); a = z W_1; y = h + gelu(a) W_2
Weights are bf16 [in, out] (W_qkv columns [q | k | v]); LayerNorm
parameters fp32.  The walk keeps the transposed weights for the forward
GEMMs (C = A B^T with B = W^T) and uses the weights as stored for the data
gradients.

Two-level activation management (Sec. 5.1): the K/V cache of the whole
sequence stays on the device; every other tensor a chunk's backward needs --
Q_i, O_i, LSE_i and the "extra planes" x_i, h_i, a_i and the two
LayerNorms' statistics -- is offloaded after the chunk's forward (all chunks
but the last by default) and prefetched before its backward.  u, z and
gelu(a) are recomputed in the backward from x, h and a.  With
``qkvol_evict`` the offloaded chunks' K/V cache rows are given up after the
forward walk as well and stream back under the last chunk's backward.

The saved tensors a chunk produces live in a region of a preallocated
device arena (ring.DeviceArena): an offloaded chunk's region is reused once
its copy has landed, and its prefetch lands in a free region.  x_i is read
from the caller's x in the forward (those rows of x are dead once
offloaded) and comes back into the chunk's region.

The host stays at most ``host_ahead`` chunk boundaries ahead of the device
(a HostPacer; 0 lets it run free).

Two options put the training operators around the blocks:
  ends=BlockEnds(...)  how a block's output b joins the residual stream, in
      one call with the LayerNorm that follows (sppo_block_norm_fwd/_bwd):
          h = alpha x + s drop(gate1 N1(O W_o)),  z = LN2(h)
          y = alpha h + s drop(gate2 N2(gelu(a) W_2))
      with a norm after the branch (or none), a gate per channel (or none),
      scales and dropout (one p for both branches and the embedding; norms before
      a branch are LayerNorms).  The masks are drawn again in the backward; b_i
      and the norms' statistics are further planes where the backward needs them.
      The forward's z comes from h before it is rounded; the backward norms the
      stored h again, whose z and statistics (they replace the kept m2, r2) serve
      dW_1 and LN2's gradient, so this z differs from the forward's by what the
      rounding of h to bf16 makes of it.
  vocab=V              the walk starts from tokens: x_i = drop(scale
      w_emb[tokens_i]), with the block ends' dropout if there are any, is
      looked up in the forward and again in the backward (it is no plane, so it
      does not travel), and dx_i becomes the table's gradient, added up over
      the reverse walk.

Only C-ABI calls and torch allocations happen here; every arithmetic step
runs in the library's kernels.
"""
from __future__ import annotations

import torch

from . import sppo as L
from .pacing import HostPacer
from .ring import DeviceArena, KeepArena, plan_capacity, plane_layout, walk_schedule

PLANES = ("x", "h", "a", "m1", "r1", "m2", "r2")  # without options

# Where a step draws masks: the offsets of its three calls, added to the step's.
DROP_EMBED, DROP_ATTN, DROP_MLP, DROP_STRIDE = 0, 1, 2, 3


class BlockEnds:
    """How the layer's two blocks join the residual stream: the norm after
    the branch ("none", "layer", "rms"), a gate per channel, the scales of the
    stream and of the branch, and the dropout's p."""

    def __init__(self, norm="none", gate=False, residual_scale=1.0, branch_scale=1.0, dropout=0.0):
        if norm not in L.NORMS:
            raise ValueError(f"unknown norm {norm!r}")
        if not 0.0 <= dropout < 1.0 or L.drop_threshold(dropout) > 65535:
            raise ValueError("dropout must be in [0, 1) and not round to 1 in units of 1/65536")
        if not L.scale_ok(residual_scale, float("inf")) or not L.scale_ok(branch_scale):
            raise ValueError("the scales must be finite, the branch's below 2^112")
        self.norm, self.gate = norm, bool(gate)
        self.residual_scale, self.branch_scale, self.dropout = residual_scale, branch_scale, dropout

    @property
    def keeps_branch(self):
        """Whether the backward needs the branch's output."""
        return self.norm != "none" or self.gate

    def params(self, n):
        """block_norm's arguments for block n (1: attention, 2: MLP) and the
        names they have among a step's parameters ([H] fp32 each); their
        gradients are out["d" + name]."""
        names = {}
        if self.norm != "none":
            names["post_gamma"] = f"g_end{n}"
        if self.norm == "layer":
            names["post_beta"] = f"b_end{n}"
        if self.gate:
            names["gate"] = f"gate{n}"
        return names


class ChunkedLayer:
    def __init__(self, S, n_chunks, Hq, Hkv, D, offsets=None, offload="none", device="cuda", eps=1e-5,
                 host_ahead=2, fwd_slots=4, ends=None, vocab=None, embed_scale=1.0):
        H = Hq * D
        wt = (Hq + 2 * Hkv) * D
        if H % 256 or wt % 256 or H > 8192:
            raise ValueError("the layer needs Hq*D and (Hq+2Hkv)*D multiples of 256 and Hq*D <= 8192")
        if vocab is not None and not 0 < vocab < 2 ** 31:
            raise ValueError("vocab must be in [1, 2^31)")
        if vocab is not None and not L.scale_ok(embed_scale):
            raise ValueError("embed_scale must be finite and below 2^112")
        self.S, self.N, self.Hq, self.Hkv, self.D, self.H, self.Wt = S, n_chunks, Hq, Hkv, D, H, wt
        self.eps = eps
        self.device = device
        self.ends, self.vocab, self.embed_scale = ends, vocab, embed_scale
        # bytes of a row of each plane: x, h, a bf16, mean/rstd of LN1, LN2 fp32;
        # with block ends their branches (bf16) and statistics
        self.row_bytes = dict(zip(PLANES, (2 * H, 2 * H, 8 * H, 4, 4, 4, 4)))
        if vocab is not None:
            del self.row_bytes["x"]
        if ends is not None and ends.keeps_branch:
            self.row_bytes.update(e1=2 * H, e2=2 * H)
        if ends is not None and ends.norm != "none":
            self.row_bytes.update(er1=4, er2=4)
        if ends is not None and ends.norm == "layer":
            self.row_bytes.update(em1=4, em2=4)
        self.planes = tuple(self.row_bytes)
        row_bytes = list(self.row_bytes.values())
        self.ctx = L.sppo_create(1, S, n_chunks, Hq, Hkv, D, dtype="bf16", chunk_offsets=offsets,
                                 offload=offload, extra_row_bytes=row_bytes)
        self.offsets = L.sppo_get_offsets(self.ctx)
        self.offload = L.OFFLOAD_MODES.get(offload, offload)
        self.s_max = max(self.offsets[i + 1] - self.offsets[i] for i in range(n_chunks))
        self.pacer = HostPacer(host_ahead)
        self.fwd_slots = fwd_slots
        self.arena = None
        self.keep = None
        self._layout = None
        self._alloc()

    def close(self):
        self.ctx.close()

    def chunk_len(self, i):
        return self.offsets[i + 1] - self.offsets[i]

    def _alloc(self):
        S, H, Wt, dev = self.S, self.H, self.Wt, self.device
        bf, f32 = torch.bfloat16, torch.float32
        HqD, HkvD, sm = self.Hq * self.D, self.Hkv * self.D, self.s_max
        e = lambda *shape, dt=bf: torch.empty(*shape, dtype=dt, device=dev)
        # the K/V cache and its gradient accumulators (full length)
        self.k, self.v = e(S, HkvD), e(S, HkvD)
        self.dk, self.dv = e(S, HkvD, dt=f32), e(S, HkvD, dt=f32)
        # transposed weights for the forward GEMMs
        self.wT = {"w_qkv": e(Wt, H), "w_o": e(H, HqD), "w_1": e(4 * H, H), "w_2": e(H, 4 * H)}
        # chunk-sized scratch
        self.u, self.z, self.g = e(sm, H), e(sm, H), e(sm, 4 * H)
        self.da, self.dz, self.dh = e(sm, 4 * H), e(sm, H), e(sm, H)
        self.dO, self.dq, self.dqkv, self.du = e(sm, HqD), e(sm, HqD), e(sm, Wt), e(sm, H)
        wsb = max(L.sppo_layernorm_bwd_workspace(self.chunk_len(i), H) for i in range(self.N))
        self.ws = torch.empty(wsb // 4, dtype=f32, device=dev)
        self.ws_bytes = wsb
        if self.ends is not None:
            self.branch, self.dbranch = e(sm, H), e(sm, H)
            probe = [L.block_norm(H, "bf16", post=self.ends.norm, pre=pre, gate_kind="channel" if self.ends.gate else
                                  "none", eps=self.eps, post_gamma=self.dk, post_beta=self.dk, gate=self.dk,
                                  pre_gamma=self.dk, pre_beta=self.dk) for pre in ("layer", "none")]
            self.ends_ws_bytes = max(L.sppo_block_norm_bwd_workspace(b, sm) for b in probe)
            self.ends_ws = torch.empty(max(self.ends_ws_bytes, 16) // 4, dtype=f32, device=dev)
        if self.vocab is not None:
            self.x, self.dx = e(sm, H), e(sm, H)
            self.emb_ws_bytes = L.sppo_embedding_bwd_workspace(sm, H)
            self.emb_ws = torch.empty(self.emb_ws_bytes // 4, dtype=f32, device=dev)

    def alloc_outputs(self):
        H, Wt, dev = self.H, self.Wt, self.device
        f32 = torch.float32
        more = {}
        if self.vocab is None:
            more["dx"] = torch.empty(self.S, H, dtype=torch.bfloat16, device=dev)
        else:
            more["dw_emb"] = torch.empty(self.vocab, H, dtype=f32, device=dev)
        if self.ends is not None:
            for n in (1, 2):
                more.update({"d" + k: torch.empty(H, dtype=f32, device=dev) for k in self.ends.params(n).values()})
        return {"y": torch.empty(self.S, H, dtype=torch.bfloat16, device=dev), **more,
                "dw_qkv": torch.empty(H, Wt, dtype=f32, device=dev),
                "dw_o": torch.empty(self.Hq * self.D, H, dtype=f32, device=dev),
                "dw_1": torch.empty(H, 4 * H, dtype=f32, device=dev),
                "dw_2": torch.empty(4 * H, H, dtype=f32, device=dev),
                **{k: torch.empty(H, dtype=f32, device=dev) for k in ("dg1", "db1", "dg2", "db2")}}

    def offload_bytes_per_row(self):
        """Bytes per token row of the offload set: Q, O, LSE, the extra planes
        (and K, V in the QKVOL modes)."""
        b = 2 * self.Hq * self.D * 2 + 4 * self.Hq + sum(self.row_bytes.values())
        if self.offload in (L.SPPO_OFFLOAD_QKVOL, L.SPPO_OFFLOAD_QKVOL_EVICT):
            b += 2 * self.Hkv * self.D * 2
        return b

    def set_offload_rows(self, rows):
        for i, r in enumerate(rows):
            L.sppo_set_offload_rows(self.ctx, i, r)

    # ------------------------------------------------------------ the walk
    def region_planes(self, i):
        """Byte sizes of chunk i's saved tensors in its arena region."""
        n, HqD = self.chunk_len(i), self.Hq * self.D
        return {"q": 2 * n * HqD, "o": 2 * n * HqD, "lse": 4 * self.Hq * n,
                **{k: n * b for k, b in self.row_bytes.items()}}

    def prepare(self, offload_chunks, lookahead):
        """Allocate the device arena and keep buffers for a walk with these
        settings (again only when they change; a walk allocates nothing).
        Returns the bytes they hold."""
        offl = tuple(sorted(set(offload_chunks)))
        key = (offl, lookahead, tuple(L.sppo_get_offload_rows(self.ctx)))
        if self._layout != key:
            self._planes = [plane_layout(self.region_planes(i)) for i in range(self.N)]
            q = self.fwd_slots - 1
            cap, q = plan_capacity(walk_schedule(self.N, offl, lookahead), [sz for _, sz in self._planes],
                                   quarantine=q)
            self.arena = None
            self.keep = None
            self.arena = DeviceArena(cap, self.device, quarantine=q)
            self.keep = KeepArena([L.sppo_keep_bytes(self.ctx, i) if i in offl else 0 for i in range(self.N)],
                                  self.device)
            self._layout = key
        return self.arena.nbytes + self.keep.nbytes

    def _acquire(self, i, s, x=None, wait=True):
        """Allocate chunk i's region; returns (offset, views of its saved
        tensors).  x_i is the caller's rows when given, else the region's x
        plane (where a prefetch puts it)."""
        off = self.arena.acquire(self.ctx, s, self._planes[i][1], i, wait)
        n, H, HqD = self.chunk_len(i), self.H, self.Hq * self.D
        bf, f32 = torch.bfloat16, torch.float32
        po = self._planes[i][0]
        pl = lambda name, shape, dt: self.arena.view(off + po[name], shape, dt)  # noqa: E731
        v = dict(q=pl("q", (n, HqD), bf), o=pl("o", (n, HqD), bf), lse=pl("lse", (self.Hq, n), f32),
                 **{k: pl(k, (n,), f32) if b == 4 else pl(k, (n, b // 2), bf) for k, b in self.row_bytes.items()
                    if k != "x"})
        v["x"] = x if x is not None else self.x[:n] if self.vocab is not None else pl("x", (n, H), bf)
        return off, v

    def _bufs(self, v, keep):
        return L.chunk_bufs(q=v["q"], o=v["o"], lse=v["lse"], k=self.k, v=self.v,
                            extra=[v[name] for name in self.planes], keep=keep)

    def _end(self, n, p, v):
        """The description of block n's end (with LN2 behind the first) and its
        statistics, for a chunk's views."""
        e = self.ends
        pre = dict(pre="layer", pre_gamma=p["g2"], pre_beta=p["b2"]) if n == 1 else {}
        bn = L.block_norm(self.H, "bf16", post=e.norm, gate_kind="channel" if e.gate else "none", eps=self.eps,
                          residual_scale=e.residual_scale, branch_scale=e.branch_scale,
                          **{k: p[name] for k, name in e.params(n).items()}, **pre)
        st = L.block_norm_stats(v.get(f"em{n}"), v.get(f"er{n}"), v["m2"] if n == 1 else None,
                                v["r2"] if n == 1 else None)
        return bn, st

    def _end_grads(self, n, out):
        g = {k: out["d" + name] for k, name in self.ends.params(n).items()}
        if n == 1:
            g.update(pre_gamma=out["dg2"], pre_beta=out["db2"])
        return L.block_norm_grads(**g)

    def step(self, inp, p, out, offload_chunks=None, lookahead=2, poison=False, stream=None, marks=None,
             ops=None, seed=0, offset=0):
        """Forward and backward of the layer over all chunks.  inp: x, dy
        [S, H] bf16 (x's chunk rows are the x planes: offloading a chunk
        makes its rows of x dead, and the prefetch brings them back into the
        chunk's arena region; poison=True overwrites every dead buffer -- the
        rows of x and the chunk's region -- with NaN once copied).  p: the
        weights (w_qkv, w_o, w_1, w_2 bf16; g1, b1, g2, b2 fp32).  marks:
        list that receives ((phase, chunk), event) at every chunk boundary.
        ops: list that receives (category, algorithmic flop, start event,
        end event) around every library call on the compute stream.  With
        vocab, inp holds tokens [S] (int32 or int64) instead of x, p w_emb
        [vocab, H] bf16, and out dw_emb instead of dx; with ends, p their
        parameters (BlockEnds.params) in fp32.  seed, offset: of the step's
        dropout, which draws at offsets offset .. offset + DROP_STRIDE - 1."""
        s = torch.cuda.current_stream() if stream is None else stream
        H, Wt, HqD, HkvD = self.H, self.Wt, self.Hq * self.D, self.Hkv * self.D
        if offload_chunks is None:
            offload_chunks = [] if self.offload == L.SPPO_OFFLOAD_NONE else list(range(self.N - 1))
        offl = set(offload_chunks)
        self.prepare(offl, lookahead)
        arena, keep = self.arena, self.keep
        arena.reset()
        ends, dy = self.ends, inp["dy"]
        x = inp["x"] if self.vocab is None else None
        drop_p = ends.dropout if ends is not None else 0.0
        if x is None:
            tokens = inp["tokens"]
            if tokens.dtype not in (torch.int32, torch.int64) or tokens.shape != (self.S,) \
                    or not tokens.is_contiguous() or not tokens.is_cuda:
                raise ValueError(f"tokens must be [{self.S}] contiguous int32 or int64 on the device")
            id_type = "i32" if tokens.dtype == torch.int32 else "i64"

        def mark(label):
            self.pacer.boundary(s)
            if marks is not None:
                ev = torch.cuda.Event(enable_timing=True)
                ev.record(s)
                marks.append((label, ev))

        def timed(cat, fn, flop=0):
            def call(*a, **kw):
                if ops is None:
                    return fn(*a, **kw)
                e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                e0.record(s)
                r = fn(*a, **kw)
                e1.record(s)
                ops.append((cat(a) if callable(cat) else cat, flop(a) if callable(flop) else flop, e0, e1))
                return r
            return call

        gemm = timed(lambda a: "gemm_" + a[0] + ("_fwd" if fwd_phase[0] and a[0] == "nt" else
                                                 "_bwd" if a[0] == "nt" else ""),
                     L.sppo_gemm_bf16, lambda a: 2 * a[1] * a[2] * a[3])
        fwd_phase = [True]
        transpose = timed("transpose", L.sppo_transpose_bf16)
        ln_fwd = timed("layernorm", L.sppo_layernorm_fwd)
        ln_bwd = timed("layernorm", L.sppo_layernorm_bwd)
        gelu = timed("gelu", L.sppo_gelu_bf16)
        pack = timed("pack", L.sppo_pack_qkv_grad)
        end_fwd = timed("block_norm", L.sppo_block_norm_fwd)
        end_bwd = timed("block_norm", L.sppo_block_norm_bwd)
        embed = timed("embedding", L.sppo_embedding_fwd)
        embed_bwd = timed("embedding", L.sppo_embedding_bwd)
        drop = lambda site, row0: L.drop_spec(drop_p, seed, offset + site, row0) if drop_p > 0 else None
        lookup = lambda n, c0: embed(n, H, self.vocab, tokens[c0:], p["w_emb"], H, self.embed_scale,
                                     drop(DROP_EMBED, c0), self.x, H, "bf16", id_type, s)
        pairs = lambda a: self.chunk_len(a[1]) * self.offsets[a[1]] + self.chunk_len(a[1]) * (self.chunk_len(a[1]) + 1) // 2
        attn_fwd = timed("attn_fwd", L.sppo_attn_fwd_chunk, lambda a: 4 * self.D * self.Hq * pairs(a))
        attn_bwd = timed("attn_bwd", L.sppo_attn_bwd_chunk, lambda a: 10 * self.D * self.Hq * pairs(a))

        mark(("wT", -1))
        transpose(p["w_qkv"], self.wT["w_qkv"], H, Wt, s)
        transpose(p["w_o"], self.wT["w_o"], HqD, H, s)
        transpose(p["w_1"], self.wT["w_1"], H, 4 * H, s)
        transpose(p["w_2"], self.wT["w_2"], 4 * H, H, s)
        held, back = {}, {}  # chunk -> (region, views): not offloaded / prefetched
        for i in range(self.N):
            mark(("fwd", i))
            n, c0 = self.chunk_len(i), self.offsets[i]
            slot, v = self._acquire(i, s, x=None if x is None else x[c0:c0 + n])
            if x is None:
                lookup(n, c0)
            u, z, g = self.u[:n], self.z[:n], self.g[:n]
            ln_fwd(n, H, v["x"], H, p["g1"], p["b1"], self.eps, u, H, v["m1"], v["r1"], s)
            wq = self.wT["w_qkv"]
            gemm("nt", n, HqD, H, u, H, wq, H, v["q"], HqD, stream=s)
            gemm("nt", n, HkvD, H, u, H, wq[HqD:], H, self.k[c0:], HkvD, stream=s)
            gemm("nt", n, HkvD, H, u, H, wq[HqD + HkvD:], H, self.v[c0:], HkvD, stream=s)
            attn_fwd(self.ctx, i, v["q"], self.k, self.v, v["o"], v["lse"], s)
            if ends is None:
                gemm("nt", n, H, HqD, v["o"], HqD, self.wT["w_o"], HqD, v["h"], H, "add_bf16", v["x"], H, stream=s)
                ln_fwd(n, H, v["h"], H, p["g2"], p["b2"], self.eps, z, H, v["m2"], v["r2"], s)
            else:
                e1, e2 = v.get("e1", self.branch), v.get("e2", self.branch)
                gemm("nt", n, H, HqD, v["o"], HqD, self.wT["w_o"], HqD, e1, H, stream=s)
                bn, st = self._end(1, p, v)
                end_fwd(bn, n, drop(DROP_ATTN, c0), v["x"], H, e1, H, v["h"], H, z, H, st, s)
            gemm("nt", n, 4 * H, H, z, H, self.wT["w_1"], H, g, 4 * H, "gelu", v["a"], 4 * H, stream=s)
            if ends is None:
                gemm("nt", n, H, 4 * H, g, 4 * H, self.wT["w_2"], 4 * H, out["y"][c0:], H, "add_bf16", v["h"], H,
                     stream=s)
            else:
                gemm("nt", n, H, 4 * H, g, 4 * H, self.wT["w_2"], 4 * H, e2, H, stream=s)
                bn, st = self._end(2, p, v)
                end_fwd(bn, n, drop(DROP_MLP, c0), v["h"], H, e2, H, out["y"][c0:], H, None, 0, st, s)
            if i in offl:
                L.sppo_offload_issue(self.ctx, i, self._bufs(v, keep.ptr(i)), s)
                arena.release(slot, after_offload=True)
                if poison:
                    # Test hook: once copied, the chunk's region and its rows of
                    # x are dead (the rows that stay went to the keep buffer).
                    L.sppo_offload_wait(self.ctx, i, s)
                    with torch.cuda.stream(s):
                        for t in v.values():
                            t.fill_(float("nan"))
            else:
                held[i] = (slot, v)
        fwd_phase[0] = False
        if self.offload == L.SPPO_OFFLOAD_QKVOL_EVICT:
            # The K/V cache rows of the offloaded chunks are given up here;
            # their copies come back on the host-to-device stream in the order
            # the last chunk's backward consumes them (chunk by chunk).
            rows = L.sppo_get_offload_rows(self.ctx)
            kv_chunks = sorted(offl, reverse=True)
            if poison:
                # Test hook: the evicted rows are dead once their copies have landed.
                for j in kv_chunks:
                    L.sppo_offload_wait(self.ctx, j, s)
                with torch.cuda.stream(s):
                    for j in kv_chunks:
                        c0 = self.offsets[j]
                        self.k[c0:c0 + rows[j]].fill_(float("nan"))
                        self.v[c0:c0 + rows[j]].fill_(float("nan"))
            for j in kv_chunks:
                L.sppo_prefetch_kv(self.ctx, j, self.k, self.v, s)
        pending = sorted(offl, reverse=True)
        nxt = 0
        for i in reversed(range(self.N)):
            while nxt < len(pending) and pending[nxt] >= i - lookahead:
                j = pending[nxt]
                slot, vj = self._acquire(j, s, wait=keep.ptr(j) is not None)
                L.sppo_prefetch(self.ctx, j, self._bufs(vj, keep.ptr(j)), s)
                back[j] = (slot, vj)
                nxt += 1
            mark(("bwd", i))
            n, c0 = self.chunk_len(i), self.offsets[i]
            slot, v = back.pop(i) if i in offl else held.pop(i)
            if i in offl:
                L.sppo_prefetch_wait(self.ctx, i, s)
            first = i == self.N - 1  # overwrite the weight gradients instead of adding
            wacc = "f32" if first else "acc_f32"
            u, z, g = self.u[:n], self.z[:n], self.g[:n]
            da, dz, dh, dO = self.da[:n], self.dz[:n], self.dh[:n], self.dO[:n]
            dyi = dy[c0:c0 + n]
            add = 0 if first else 1
            dres, dbr = dyi, dyi  # gradients of h (along the stream) and of the MLP's output
            if ends is not None:
                # y = alpha h + s drop(gate2 N2(e2))
                dres, dbr = dh, self.dbranch
                bn, st = self._end(2, p, v)
                end_bwd(bn, n, drop(DROP_MLP, c0), v.get("e2"), H, None, 0, st, None, 0, dyi, H, dres, H, dbr, H,
                        self._end_grads(2, out), self.ends_ws, self.ends_ws_bytes, add, s)
            # y = h + gelu(a) W2
            gelu(v["a"], g, n * 4 * H, s)
            gemm("nt", n, 4 * H, H, dbr, H, p["w_2"], H, da, 4 * H, "dgelu", v["a"], 4 * H, stream=s)
            gemm("tn", 4 * H, H, n, g, 4 * H, dbr, H, out["dw_2"], H, wacc, stream=s)
            # a = z W1, z = LN2(h)
            ln_fwd(n, H, v["h"], H, p["g2"], p["b2"], self.eps, z, H, v["m2"], v["r2"], s)
            gemm("nt", n, H, 4 * H, da, 4 * H, p["w_1"], 4 * H, dz, H, stream=s)
            gemm("tn", H, 4 * H, n, z, H, da, 4 * H, out["dw_1"], 4 * H, wacc, stream=s)
            if ends is None:
                ln_bwd(n, H, v["h"], H, p["g2"], v["m2"], v["r2"], dz, H, dyi, H, dh, H, out["dg2"],
                                     out["db2"], self.ws, self.ws_bytes, accumulate=0 if first else 1, stream=s)
                dbr = dh
            else:
                # h = alpha x + s drop(gate1 N1(e1)), z = LN2(h); dh: from h's gradient to x's
                bn, st = self._end(1, p, v)
                end_bwd(bn, n, drop(DROP_ATTN, c0), v.get("e1"), H, v["h"], H, st, dz, H, dres, H, dh, H, dbr, H,
                        self._end_grads(1, out), self.ends_ws, self.ends_ws_bytes, add, s)
            # h = x + O Wo
            gemm("nt", n, HqD, H, dbr, H, p["w_o"], H, dO, HqD, stream=s)
            gemm("tn", HqD, H, n, v["o"], HqD, dbr, H, out["dw_o"], H, wacc, stream=s)
            attn_bwd(self.ctx, i, v["q"], self.k, self.v, v["o"], v["lse"], dO, self.dq[:n],
                                  self.dk, self.dv, s)
            # q, k, v = u W_qkv (chunk i's dK/dV rows are complete now)
            dqkv = self.dqkv[:n]
            pack(n, HqD, HkvD, self.dq[:n], self.dk, self.dv, c0, dqkv, s)
            if x is None:
                lookup(n, c0)
            ln_fwd(n, H, v["x"], H, p["g1"], p["b1"], self.eps, u, H, v["m1"], v["r1"], s)
            gemm("nt", n, H, Wt, dqkv, Wt, p["w_qkv"], Wt, self.du[:n], H, stream=s)
            gemm("tn", H, Wt, n, u, H, dqkv, Wt, out["dw_qkv"], Wt, wacc, stream=s)
            # u = LN1(x); x also reaches h
            dxi = self.dx if x is None else out["dx"][c0:]
            ln_bwd(n, H, v["x"], H, p["g1"], v["m1"], v["r1"], self.du[:n], H, dh, H,
                                 dxi, H, out["dg1"], out["db1"], self.ws, self.ws_bytes,
                                 accumulate=0 if first else 1, stream=s)
            if x is None:
                embed_bwd(n, H, self.vocab, tokens[c0:], dxi, H, self.embed_scale, drop(DROP_EMBED, c0),
                          out["dw_emb"], H, self.emb_ws, self.emb_ws_bytes, add, "bf16", id_type, s)
            arena.release(slot)
        mark(("end", -1))

    @staticmethod
    def flops(S, offsets, Hq, Hkv, D):
        """Algorithmic flop of one forward + backward: the GEMMs (3 x 2 m n k
        per projection) plus attention (14 D per visible pair per head)."""
        H, wt = Hq * D, (Hq + 2 * Hkv) * D
        gemm = 3 * 2 * S * (H * wt + Hq * D * H + 2 * H * 4 * H)
        pairs = 0
        for i in range(len(offsets) - 1):
            s_i, c_i = offsets[i + 1] - offsets[i], offsets[i]
            pairs += s_i * c_i + s_i * (s_i + 1) // 2
        return gemm + 14 * D * Hq * pairs, gemm
