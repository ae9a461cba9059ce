"""Timed cases of the training operators around a chunk's attention: dropout
whose mask is drawn again from a counter, the norms, gate and residual at a
block's two ends, and the embedding with its gradient by sorted tokens.

``own`` selects the side: False computes each operator from elementary torch
operations in fp32, True makes the library's calls.  The sizes are those of
the package's layer (hidden size 4096, chunks of 8192 tokens), of its tests
(widths from 64 to 8192, ragged row counts) and generic ones between them.

The operators, for global row t = row0 + r, column c, row width W:
    keep(t, c)  16 random bits u of element e = t W + c, keep when u >= T with
                T = round(65536 p); a kept value is scaled by 65536 / (65536 - T).
                u: half word e % 8 (low halves first) of Philox4x32-10 with
                counter (e / 8, offset) and key seed.
    dropout     y = res + keep * x
    block norm  h = alpha x + s keep (g * N_post(b)),  z = N_pre(h)
    embedding   y = keep * (s table[id]); ids outside the table give zeros
and their gradients.
"""
import math

import numpy as np
import torch

own = False

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DT = {"bf16": BF, "f32": F32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5


# ------------------------------------------------------------------- the cases
def _dropout(name, rows, W, dtype="bf16", pad=0, res=False, p=0.1, row0=0):
    return {"name": name, "kind": "dropout", "rows": rows, "W": W, "dtype": dtype, "pad": pad, "res": res, "p": p,
            "row0": row0}


def _norm(name, kind, rows, W, dtype="bf16", post="layer", pre="layer", gate="none", p=0.0, alpha=1.0, scale=1.0,
          pad=0):
    return {"name": name, "kind": kind, "rows": rows, "W": W, "dtype": dtype, "post": post, "pre": pre, "gate": gate,
            "p": p, "alpha": alpha, "scale": scale, "pad": pad}


def _embed(name, kind, rows, W, V, chunks=1, dtype="bf16", ids="i64", p=0.0, scale=1.0, padded=0):
    return {"name": name, "kind": kind, "rows": rows, "W": W, "V": V, "chunks": chunks, "dtype": dtype, "ids": ids,
            "p": p, "scale": scale, "padded": padded}


def listed():
    return [
        # One token's activations: launch latency.
        _dropout("dropout_1x4096", 1, 4096),
        # A chunk's branch output added to the residual stream, as at the end of each block.
        _dropout("dropout_residual_8k", 8192, 4096, res=True),
        # A strided fp32 activation far into a long sequence (element indices past 32 bits).
        _dropout("dropout_f32_strided", 5001, 1024, "f32", pad=8, p=0.25, row0=9000000),
        # A short fp32 check run of the block boundary, norms on both sides.
        _norm("norm_fwd_f32_37x256", "norm_fwd", 37, 256, "f32", gate="channel", p=0.1),
        # The boundary of a chunk of the layer configuration: both LayerNorms, a gate per channel, dropout.
        _norm("norm_fwd_8k", "norm_fwd", 8192, 4096, gate="channel", p=0.1, alpha=1.0, scale=0.5),
        # The same boundary with RMS norms and a gate per token on a ragged chunk, wide rows, no dropout.
        _norm("norm_fwd_rms_3001x8192", "norm_fwd", 3001, 8192, post="rms", pre="rms", gate="token", alpha=0.9),
        # Its backward on a chunk of the layer configuration.
        _norm("norm_bwd_8k", "norm_bwd", 8192, 4096, gate="channel", p=0.1, alpha=1.0, scale=0.5),
        # A pre-norm block's backward (no norm after the branch) of a small layer on a ragged chunk.
        _norm("norm_bwd_prenorm_5001x1024", "norm_bwd", 5001, 1024, post="none", p=0.1),
        # Few wide fp32 rows with RMS norms and a gate per token.
        _norm("norm_bwd_rms_f32_130x8192", "norm_bwd", 130, 8192, "f32", post="rms", pre="rms", gate="token", p=0.2,
              alpha=0.9),
        # The tokens of a chunk of the layer configuration, scaled, with dropout on the embedding.
        _embed("embed_fwd_8k", "embed_fwd", 8192, 4096, 32768, p=0.1, scale=64.0),
        # The table gradient over two chunks of 8192 of the reverse walk: the first overwrites, the second adds.
        _embed("embed_bwd_16k", "embed_bwd", 16384, 4096, 32768, chunks=2, p=0.1, scale=64.0),
        # One long ragged chunk of a narrow layer, padded at its end.
        _embed("embed_bwd_65521x1024", "embed_bwd", 65521, 1024, 50001, ids="i32", padded=1500),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("dropout", "norm_fwd", "norm_fwd", "norm_bwd", "norm_bwd", "norm_bwd", "embed_fwd",
                       "embed_bwd", "embed_bwd"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    W = 8 * _log(rng, 8, 1024)
    rows = _log(rng, 1, 16384)
    p = rng.choice((0.0, 0.1, 0.3))
    if kind == "dropout":
        c = _dropout(None, rows, W, dtype, rng.choice((0, 0, 8, 24)), rng.random() < 0.5, rng.uniform(0.01, 0.6),
                     rng.choice((0, 12345, 7000000)))
    elif kind in ("norm_fwd", "norm_bwd"):
        post, pre = rng.choice((("layer", "layer"), ("rms", "rms"), ("none", "layer"), ("none", "rms"),
                                ("layer", "none"), ("rms", "layer")))
        c = _norm(None, kind, rows, W, dtype, post, pre, rng.choice(("none", "channel", "token")), p,
                  rng.choice((1.0, 0.8)), rng.choice((1.0, 0.25)), rng.choice((0, 0, 8)))
    else:
        c = _embed(None, kind, rows, W, _log(rng, 300, 60000), rng.randint(1, min(3, rows)) if kind == "embed_bwd" else 1,
                   dtype, rng.choice(("i32", "i64")), p, rng.choice((1.0, 32.0)), rng.choice((0, 0, rows // 5)))
    del c["name"]
    limit = 6 * 8192 * 4096
    while c["rows"] > c.get("chunks", 1) and work(c)["bytes"] > limit:
        c["rows"] = max(c.get("chunks", 1), c["rows"] * 3 // 4)
        if "padded" in c:
            c["padded"] = min(c["padded"], c["rows"] // 5)
    while work(c)["bytes"] > limit and c.get("V", 0) > 300:
        c["V"] = max(300, c["V"] * 3 // 4)
    return c


# ------------------------------------------------------------------- the inputs
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + salt)


def _randn(rows, W, pad, dtype, g, scale=1.0, shift=0.0):
    x = torch.randn(rows, W + pad, generator=g, device="cuda") * scale + shift
    return x.to(DT[dtype])[:, :W]


def _stats(x, norm):
    """(mean, rstd) of the rows, as the forward keeps them."""
    x = x.to(F64)
    mean = x.mean(dim=1) if norm == "layer" else torch.zeros(x.shape[0], dtype=F64, device=x.device)
    var = ((x - mean[:, None]) ** 2).mean(dim=1)
    return mean.to(F32), (1.0 / torch.sqrt(var + EPS)).to(F32)


def _bounds(case):
    rows, n = case["rows"], case["chunks"]
    return [rows * i // n for i in range(n + 1)]


def prepare(case, seed):
    kind, rows, W = case["kind"], case["rows"], case["W"]
    dt = DT[case["dtype"]]
    st = {"case": case, "seed": 7919 * seed + 12345678901, "offset": 3 * seed + 5}
    e = lambda *shape, t=dt: torch.empty(*shape, dtype=t, device="cuda")
    if kind == "dropout":
        st["x"] = _randn(rows, W, case["pad"], case["dtype"], _gen(seed, 1))
        st["res"] = _randn(rows, W, case["pad"], case["dtype"], _gen(seed, 2), 2.0) if case["res"] else None
        st["y"] = e(rows, W + case["pad"])[:, :W]
    elif kind in ("norm_fwd", "norm_bwd"):
        g = _gen(seed, 3)
        chan = 1.0 + torch.rand(W, generator=g, device="cuda") * 3.0  # channels of unequal size
        st["b"] = _randn(rows, W, case["pad"], case["dtype"], g)
        st["b"].mul_(chan.to(dt))
        for name in ("post", "pre"):
            st[name + "_gamma"] = st[name + "_beta"] = None
            if case[name] != "none":
                st[name + "_gamma"] = 1.0 + 0.1 * torch.randn(W, generator=g, device="cuda")
                if case[name] == "layer":
                    st[name + "_beta"] = 0.1 * torch.randn(W, generator=g, device="cuda")
        n_gate = {"none": 0, "channel": W, "token": rows}[case["gate"]]
        st["gate"] = torch.rand(n_gate, generator=g, device="cuda") + 0.25 if n_gate else None
        if kind == "norm_fwd":
            st["x"] = _randn(rows, W, case["pad"], case["dtype"], g, 2.0, 0.25)
        else:
            st["h"] = _randn(rows, W, case["pad"], case["dtype"], g, 2.0, 0.25)
            st["post_mean"], st["post_rstd"] = _stats(st["b"], case["post"])
            st["pre_mean"], st["pre_rstd"] = _stats(st["h"], case["pre"])
            st["dz"] = _randn(rows, W, case["pad"], case["dtype"], g, 0.1) if case["pre"] != "none" else None
            st["dh"] = _randn(rows, W, case["pad"], case["dtype"], g, 0.1)
    else:
        g = _gen(seed, 4)
        V = case["V"]
        # Token frequencies fall as one over the rank.
        u = torch.rand(rows, generator=g, device="cuda", dtype=F64)
        ids = (torch.exp(u * math.log(V + 1.0)).to(torch.int64) - 1).clamp_(0, V - 1)
        if case["padded"]:
            ids[rows - case["padded"]:] = -1
        st["ids"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        if kind == "embed_fwd":
            st["table"] = _randn(V, W, 0, case["dtype"], g, 0.02)
            st["y"] = e(rows, W)
        else:
            st["dy"] = _randn(rows, W, 0, case["dtype"], g, 0.1)
    if own:
        _plan(st)
    return st


# ------------------------------------------------------------------- plain form
def _philox(rows, W, row0, seed, offset):
    """[rows, W] 16-bit draws as int64, Philox4x32-10; the 64-bit products are
    formed from 16-bit halves (int64 holds them)."""
    M = 0xFFFFFFFF
    e = torch.arange(rows * (W // 8), dtype=torch.int64, device="cuda") + row0 * (W // 8)
    c = [e & M, (e >> 32) & M, torch.full_like(e, offset & M), torch.full_like(e, (offset >> 32) & M)]
    k0, k1 = seed & M, (seed >> 32) & M

    def mul(a, x):
        lo, hi = a * (x & 0xFFFF), a * (x >> 16)
        t = hi + (lo >> 16)
        return (t >> 16) & M, ((t & 0xFFFF) << 16) | (lo & 0xFFFF)

    for _ in range(10):
        h0, l0 = mul(0xD2511F53, c[0])
        h1, l1 = mul(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
    u = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], dim=1)
    return u.reshape(rows, W)


def _drop(x, case, st, row0):
    """keep * x / (1 - p), the mask drawn from the elements' positions."""
    T = int(math.floor(case["p"] * 65536.0 + 0.5))
    if T == 0:
        return x
    u = _philox(x.shape[0], x.shape[1], row0, st["seed"], st["offset"])
    return torch.where(u >= T, x * (65536.0 / (65536.0 - T)), torch.zeros((), dtype=x.dtype, device=x.device))


def _center(x, norm, eps=EPS):
    mean = x.mean(dim=1) if norm == "layer" else torch.zeros(x.shape[0], dtype=x.dtype, device=x.device)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(dim=1) + eps)
    return d * rstd[:, None], mean, rstd


def _affine(xhat, gamma, beta):
    y = xhat * gamma
    return y if beta is None else y + beta


def _gated(n, case, st):
    if case["gate"] == "channel":
        return n * st["gate"]
    return n * st["gate"][:, None] if case["gate"] == "token" else n


def _norm_back(g, xhat, rstd, norm):
    """Gradient at a norm's input from the gradient g at xhat."""
    m2 = (g * xhat).mean(dim=1, keepdim=True)
    d = g - xhat * m2
    if norm == "layer":
        d = d - g.mean(dim=1, keepdim=True)
    return d * rstd[:, None]


def _run_plain(st):
    case = st["case"]
    kind, dt = case["kind"], DT[case["dtype"]]
    if kind == "dropout":
        y = _drop(st["x"].to(F32), case, st, case["row0"])
        if case["res"]:
            y = y + st["res"].to(F32)
        return {"y": y.to(dt)}
    if kind == "norm_fwd":
        n, out = st["b"].to(F32), {}
        if case["post"] != "none":
            xhat, out["post_mean"], out["post_rstd"] = _center(n, case["post"])
            n = _affine(xhat, st["post_gamma"], st["post_beta"])
        h = case["alpha"] * st["x"].to(F32) + case["scale"] * _drop(_gated(n, case, st), case, st, 0)
        out["h"] = h.to(dt)
        if case["pre"] != "none":
            xhat, out["pre_mean"], out["pre_rstd"] = _center(h, case["pre"])
            out["z"] = _affine(xhat, st["pre_gamma"], st["pre_beta"]).to(dt)
        return {k: v for k, v in out.items() if not (k[-4:] == "mean" and case[k[:-5]] == "rms")}
    if kind == "norm_bwd":
        out, D = {}, st["dh"].to(F32)
        if case["pre"] != "none":
            xhat, dz = (st["h"].to(F32) - st["pre_mean"][:, None]) * st["pre_rstd"][:, None], st["dz"].to(F32)
            out["dpre_gamma"] = (dz * xhat).sum(dim=0)
            if case["pre"] == "layer":
                out["dpre_beta"] = dz.sum(dim=0)
            D = D + _norm_back(dz * st["pre_gamma"], xhat, st["pre_rstd"], case["pre"])
        out["dx"] = (case["alpha"] * D).to(dt)
        m = case["scale"] * _drop(D, case, st, 0)
        n = st["b"].to(F32)
        if case["post"] != "none":
            bhat = (n - st["post_mean"][:, None]) * st["post_rstd"][:, None]
            n = _affine(bhat, st["post_gamma"], st["post_beta"])
        if case["gate"] != "none":
            out["dgate"] = (m * n).sum(dim=0 if case["gate"] == "channel" else 1)
        dn = _gated(m, case, st)
        if case["post"] != "none":
            out["dpost_gamma"] = (dn * bhat).sum(dim=0)
            if case["post"] == "layer":
                out["dpost_beta"] = dn.sum(dim=0)
            dn = _norm_back(dn * st["post_gamma"], bhat, st["post_rstd"], case["post"])
        out["db"] = dn.to(dt)
        return out
    ids = st["ids"].to(torch.int64)
    ok = (ids >= 0) & (ids < case["V"])
    if kind == "embed_fwd":
        y = case["scale"] * st["table"][ids.clamp(0, case["V"] - 1)].to(F32)
        return {"y": (_drop(y, case, st, 0) * ok[:, None]).to(dt)}
    dw = torch.zeros(case["V"], case["W"], device="cuda")
    b = _bounds(case)
    for i in reversed(range(case["chunks"])):
        r = slice(b[i], b[i + 1])
        g = case["scale"] * _drop(st["dy"][r].to(F32), case, st, b[i])
        dw.index_add_(0, ids[r].clamp(0, case["V"] - 1), g * ok[r][:, None])
    return {"dtable": dw}


# ------------------------------------------------------------------- the library's calls
def _plan(st):
    """What a program sets up once: the output buffers, the workspaces, the
    descriptions of the norms and of the dropout."""
    from paper_2503_10377_amd import sppo as L

    case = st["case"]
    kind, rows, W, dt = case["kind"], case["rows"], case["W"], DT[case["dtype"]]
    e = lambda *shape, t=F32: torch.empty(*shape, dtype=t, device="cuda")
    st["L"] = L
    spec = lambda row0: L.drop_spec(case["p"], st["seed"], st["offset"], row0) if case["p"] > 0 else None
    st["drop"] = spec(case.get("row0", 0))
    if kind in ("norm_fwd", "norm_bwd"):
        st["bn"] = L.block_norm(W, case["dtype"], post=case["post"], pre=case["pre"], gate_kind=case["gate"], eps=EPS,
                                residual_scale=case["alpha"], branch_scale=case["scale"], post_gamma=st["post_gamma"],
                                post_beta=st["post_beta"], gate=st["gate"], pre_gamma=st["pre_gamma"],
                                pre_beta=st["pre_beta"])
        act = lambda: e(rows, W + case["pad"], t=dt)[:, :W]
        out = {}
        if kind == "norm_fwd":
            out["h"] = act()
            if case["pre"] != "none":
                out["z"] = act()
            for k in ("post", "pre"):
                if case[k] == "layer":
                    out[k + "_mean"] = e(rows)
                if case[k] != "none":
                    out[k + "_rstd"] = e(rows)
            st["stats"] = L.block_norm_stats(*(out.get(k) for k in ("post_mean", "post_rstd", "pre_mean", "pre_rstd")))
        else:
            out["dx"], out["db"] = act(), act()
            for k in ("post", "pre"):
                if case[k] != "none":
                    out[f"d{k}_gamma"] = e(W)
                if case[k] == "layer":
                    out[f"d{k}_beta"] = e(W)
            if st["gate"] is not None:
                out["dgate"] = torch.empty_like(st["gate"])
            st["stats"] = L.block_norm_stats(st["post_mean"], st["post_rstd"], st["pre_mean"], st["pre_rstd"])
            st["grads"] = L.block_norm_grads(out.get("dpost_gamma"), out.get("dpost_beta"), out.get("dgate"),
                                             out.get("dpre_gamma"), out.get("dpre_beta"))
            st["ws_bytes"] = L.sppo_block_norm_bwd_workspace(st["bn"], rows)
            st["ws"] = e(max(1, st["ws_bytes"] // 4))
        st["out"] = out
    elif kind == "embed_bwd":
        b = _bounds(case)
        st["dtable"] = e(case["V"], W)
        st["ws_bytes"] = max(L.sppo_embedding_bwd_workspace(b[i + 1] - b[i], W) for i in range(case["chunks"]))
        st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, device="cuda")
        st["drops"] = [spec(b[i]) for i in range(case["chunks"])]


def _run_own(st):
    case, L = st["case"], st["L"]
    kind, rows, W, dtype = case["kind"], case["rows"], case["W"], case["dtype"]
    ld = W + case.get("pad", 0)
    if kind == "dropout":
        L.sppo_dropout(rows, W, st["x"], ld, st["drop"], st["y"], ld, res=st["res"], ldres=ld, dtype=dtype)
        return {"y": st["y"]}
    if kind == "norm_fwd":
        out = st["out"]
        L.sppo_block_norm_fwd(st["bn"], rows, st["drop"], st["x"], ld, st["b"], ld, out["h"], ld, out.get("z"), ld,
                              st["stats"])
        return out
    if kind == "norm_bwd":
        out = st["out"]
        L.sppo_block_norm_bwd(st["bn"], rows, st["drop"], st["b"], ld, st["h"], ld, st["stats"], st["dz"], ld,
                              st["dh"], ld, out["dx"], ld, out["db"], ld, st["grads"], st["ws"], st["ws_bytes"],
                              accumulate=0)
        return out
    if kind == "embed_fwd":
        L.sppo_embedding_fwd(rows, W, case["V"], st["ids"], st["table"], W, case["scale"], st["drop"], st["y"], W,
                             dtype=dtype, id_type=case["ids"])
        return {"y": st["y"]}
    b, n = _bounds(case), case["chunks"]
    for i in reversed(range(n)):
        L.sppo_embedding_bwd(b[i + 1] - b[i], W, case["V"], st["ids"][b[i]:], st["dy"][b[i]:], W, case["scale"],
                             st["drops"][i], st["dtable"], W, st["ws"], st["ws_bytes"],
                             accumulate=0 if i == n - 1 else 1, dtype=dtype, id_type=case["ids"])
    return {"dtable": st["dtable"]}


def _ordered(out):
    return {k: out[k] for k in sorted(out)}


def run(state):
    return _ordered(_run_own(state) if own else _run_plain(state))


# ------------------------------------------------------------------- work
def work(case):
    """Bytes: each input read once, each output written once.  Flops: the
    multiplications and additions of the formulas; a draw counts as 20 wide
    products for eight elements."""
    kind, rows, W = case["kind"], case["rows"], case["W"]
    n, el = rows * W, SIZE[case["dtype"]]
    rnd = 2.5 * n if case["p"] > 0 else 0
    if kind == "dropout":
        return {"bytes": n * el * (3 if case["res"] else 2), "flops": rnd + n * (2 if case["res"] else 1)}
    norms = sum(case.get(k, "none") != "none" for k in ("post", "pre"))
    if kind == "norm_fwd":
        return {"bytes": n * el * (4 if case["pre"] != "none" else 3), "flops": rnd + n * (4 + 7 * norms)}
    if kind == "norm_bwd":
        # b is needed for its norm's or its gate's gradient, h and dz for the norm in front of the next block.
        reads = 1 + (2 if case["pre"] != "none" else 0) + (1 if case["post"] != "none" or case["gate"] != "none" else 0)
        return {"bytes": n * el * (reads + 2), "flops": rnd + n * (4 + 12 * norms)}
    idb = 4 if case["ids"] == "i32" else 8
    live = rows - case["padded"]
    if kind == "embed_fwd":
        # Distinct rows of the table are read once: their expected number under p(rank) ~ 1 / rank.
        return {"bytes": rows * idb + n * el + int(_distinct(live, case["V"])) * W * el, "flops": rnd + n}
    return {"bytes": rows * idb + live * W * el + case["V"] * W * 4, "flops": rnd + 2 * n}


def _distinct(rows, V):
    k = np.arange(1, V + 1, dtype=np.float64)
    q = np.log1p(1.0 / k) / math.log(V + 1.0)
    return float((-np.expm1(rows * np.log1p(-q))).sum())


# ------------------------------------------------------------------- 64-bit values
def _keep64(rows, W, row0, seed, offset, p):
    """Scaled keep factors [rows, W] in fp64: the generator in NumPy's unsigned
    64-bit products."""
    T = int(math.floor(p * 65536.0 + 0.5))
    if T == 0:
        return None
    mask = np.uint64(0xFFFFFFFF)
    sh = np.uint64(32)
    idx = np.arange(row0 * W // 8, (row0 + rows) * W // 8, dtype=np.uint64)
    x0, x1 = idx & mask, idx >> sh
    x2 = np.full_like(idx, offset & 0xFFFFFFFF)
    x3 = np.full_like(idx, offset >> 32)
    ka, kb = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        pa, pb = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (pb >> sh) ^ x1 ^ np.uint64(ka), pb & mask, (pa >> sh) ^ x3 ^ np.uint64(kb), pa & mask
        ka, kb = (ka + 0x9E3779B9) % 2 ** 32, (kb + 0xBB67AE85) % 2 ** 32
    words = np.stack([x0, x1, x2, x3], axis=1).astype("<u4")
    kept = words.view("<u2").reshape(rows, W) >= T
    return torch.from_numpy(kept).cuda().to(F64) * (65536.0 / (65536 - T))


def exact(case, seed):
    return _ordered(_exact(case, seed))


def _exact(case, seed):
    st = prepare(case, seed)
    kind, rows, W = case["kind"], case["rows"], case["W"]
    k = _keep64(rows, W, case.get("row0", 0), st["seed"], st["offset"], case["p"])
    k = 1.0 if k is None else k
    d = lambda t: t.to(F64)
    if kind == "dropout":
        y = d(st["x"]) * k
        return {"y": y + d(st["res"]) if case["res"] else y}
    if kind == "norm_fwd":
        out = {}
        v = d(st["b"])

        def norm(v, name):
            mu = v.mean(1, keepdim=True) if case[name] == "layer" else torch.zeros_like(v[:, :1])
            rs = (((v - mu) ** 2).mean(1, keepdim=True) + EPS) ** -0.5
            if case[name] == "layer":
                out[name + "_mean"] = mu[:, 0]
            out[name + "_rstd"] = rs[:, 0]
            y = (v - mu) * rs * d(st[name + "_gamma"])
            return y + d(st[name + "_beta"]) if case[name] == "layer" else y

        if case["post"] != "none":
            v = norm(v, "post")
        if case["gate"] != "none":
            v = v * (d(st["gate"]) if case["gate"] == "channel" else d(st["gate"])[:, None])
        h = case["alpha"] * d(st["x"]) + case["scale"] * (v * k)
        if case["pre"] != "none":
            out["z"] = norm(h, "pre")
        out["h"] = h
        return out
    if kind == "norm_bwd":
        out = {}
        total = d(st["dh"])

        def through(name, at, grad):
            """Gradient at the norm's input; the parameters' into out."""
            rs = d(st[name + "_rstd"])[:, None]
            hat = (at - d(st[name + "_mean"])[:, None]) * rs if case[name] == "layer" else at * rs
            out[f"d{name}_gamma"] = (grad * hat).sum(0)
            if case[name] == "layer":
                out[f"d{name}_beta"] = grad.sum(0)
            w = grad * d(st[name + "_gamma"])
            back = w - hat * (w * hat).sum(1, keepdim=True) / W
            if case[name] == "layer":
                back = back - w.sum(1, keepdim=True) / W
            return back * rs, hat

        if case["pre"] != "none":
            total = total + through("pre", d(st["h"]), d(st["dz"]))[0]
        out["dx"] = case["alpha"] * total
        m = case["scale"] * total * k
        gate = {"none": lambda: 1.0, "channel": lambda: d(st["gate"]), "token": lambda: d(st["gate"])[:, None]}
        gate = gate[case["gate"]]()
        n = d(st["b"])
        if case["post"] != "none":
            out["db"], hat = through("post", n, m * gate)
            n = hat * d(st["post_gamma"])
            if case["post"] == "layer":
                n = n + d(st["post_beta"])
        else:
            out["db"] = m * gate
        if case["gate"] != "none":
            out["dgate"] = (m * n).sum(0 if case["gate"] == "channel" else 1)
        return out
    ids = st["ids"].long()
    inside = (ids >= 0) & (ids < case["V"])
    if kind == "embed_fwd":
        y = torch.zeros(rows, W, dtype=F64, device="cuda")
        y[inside] = case["scale"] * d(st["table"])[ids[inside]]
        return {"y": y * k}
    g = case["scale"] * d(st["dy"]) * k
    dw = torch.zeros(case["V"], W, dtype=F64, device="cuda")
    dw.index_put_((ids[inside],), g[inside], accumulate=True)
    return {"dtable": dw}
