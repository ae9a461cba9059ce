"""fp64 oracle of the training operators around the layer: dropout from a
counter-based generator, the norms, gate and residual at a block's end, and
the token embedding; forward and analytic gradient.

TEST INFRASTRUCTURE ONLY -- never imported by the product path.

With t the global row (row0 + r), c the column and W the row's width:
    keep     u = half word e % 8 of Philox4x32-10(counter (e // 8, offset), key
             seed), e = t W + c; 65536 / (65536 - T) where u >= T, else 0, with
             T = round(65536 p)
    norm     LayerNorm (v - mean) rstd gamma + beta, RMSNorm v rstd gamma + beta
    block    n = N_post(b); h = alpha x + s keep (g n); z = N_pre(h)
    lookup   y = keep (s table[id]), zero for ids outside the table
    layer    the layer of transformer_layer whose two branches join the stream
             by block (LN2 the norm behind the first, none behind the second)

Pins (tests/test_train_ops_cpu.py): the generator's published answers; the
drawn share of kept elements; central differences of every gradient; the
lookup's gradient as the transpose of the lookup.
"""
from __future__ import annotations

import math

import numpy as np

from .causal_attention import attention_bwd, attention_fwd
from .transformer_layer import gelu, gelu_grad, layer_norm, layer_norm_bwd

_U32 = 0xFFFFFFFF


def _f64(x):
    return np.asarray(x, dtype=np.float64)


def philox4x32(counter, key, rounds=10):
    """Philox4x32 of Salmon, Moraes, Dror and Shaw (SC 2011), section 3: four
    counter words [..., 4] and two key words to four output words."""
    c = np.asarray(counter, dtype=np.uint64)
    k = [int(key[0]), int(key[1])]
    x = [c[..., i] for i in range(4)]
    s32, m = np.uint64(32), np.uint64(_U32)
    for _ in range(rounds):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> s32) ^ x[1] ^ np.uint64(k[0]), b & m, (a >> s32) ^ x[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & _U32, (k[1] + 0xBB67AE85) & _U32]
    return np.stack(x, axis=-1)


def threshold(p) -> int:
    return int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))


def keep_factor(rows, W, p, seed, offset=0, row0=0):
    """[rows, W]: the factor of every element, 0 or 1 / (drawn probability)."""
    T = threshold(p)
    g = row0 * (W // 8) + np.arange(rows * (W // 8), dtype=object if row0 * W >= 2 ** 62 else np.int64)
    ctr = np.stack([(g & _U32).astype(np.uint64), (g >> 32).astype(np.uint64),
                    np.full(len(g), offset & _U32, dtype=np.uint64), np.full(len(g), offset >> 32, dtype=np.uint64)],
                   axis=-1)
    w = philox4x32(ctr, (seed & _U32, seed >> 32))
    u = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], axis=-1).reshape(rows, W)
    return np.where(u >= T, 65536.0 / (65536.0 - T), 0.0)


def drop(x, keep):
    """keep * x with a dropped element zero whatever its value."""
    return np.where(keep > 0, _f64(x) * keep, 0.0)


def norm_stats(v, kind, eps):
    v = _f64(v)
    mean = v.mean(axis=1) if kind == "layer" else np.zeros(len(v))
    return mean, 1.0 / np.sqrt(((v - mean[:, None]) ** 2).mean(axis=1) + eps)


def _hat(v, mean, rstd):
    return (_f64(v) - _f64(mean)[:, None]) * _f64(rstd)[:, None]


def _gate(kind, gate):
    return {"none": lambda: 1.0, "channel": lambda: _f64(gate)[None, :], "token": lambda: _f64(gate)[:, None]}[kind]()


def block_norm_fwd(x, b, cfg, par, keep):
    """cfg: post, pre ("none", "layer", "rms"), gate ("none", "channel",
    "token"), eps, alpha, scale.  par: post_gamma, post_beta, gate, pre_gamma,
    pre_beta (absent or None where there is none).  Returns h, z and stats."""
    out = {}
    n = _f64(b)
    if cfg["post"] != "none":
        out["post_mean"], out["post_rstd"] = norm_stats(n, cfg["post"], cfg["eps"])
        n = _hat(n, out["post_mean"], out["post_rstd"]) * _f64(par["post_gamma"])
        if par.get("post_beta") is not None:
            n = n + _f64(par["post_beta"])
    h = cfg["alpha"] * _f64(x) + cfg["scale"] * drop(_gate(cfg["gate"], par.get("gate")) * n, keep)
    out["h"] = h
    if cfg["pre"] != "none":
        out["pre_mean"], out["pre_rstd"] = norm_stats(h, cfg["pre"], cfg["eps"])
        out["z"] = _hat(h, out["pre_mean"], out["pre_rstd"]) * _f64(par["pre_gamma"])
        if par.get("pre_beta") is not None:
            out["z"] = out["z"] + _f64(par["pre_beta"])
    return out


def _norm_bwd(v, mean, rstd, g, kind):
    """Gradient at the norm's input from g at the normalised value."""
    vh = _hat(v, mean, rstd)
    d = g - vh * (g * vh).mean(axis=1, keepdims=True)
    if kind == "layer":
        d = d - g.mean(axis=1, keepdims=True)
    return d * _f64(rstd)[:, None]


def block_norm_bwd(b, h, stats, dz, dh, cfg, par, keep):
    """Gradients of sum(dz z) + sum(dh h) at x, b and the parameters, from the
    kept b, h and statistics (dz None where there is no z, dh None: zero)."""
    out = {}
    D = np.zeros(keep.shape) if dh is None else _f64(dh)
    if cfg["pre"] != "none":
        hh = _hat(h, stats["pre_mean"], stats["pre_rstd"])
        out["pre_gamma"], out["pre_beta"] = (_f64(dz) * hh).sum(axis=0), _f64(dz).sum(axis=0)
        D = D + _norm_bwd(h, stats["pre_mean"], stats["pre_rstd"], _f64(dz) * _f64(par["pre_gamma"]), cfg["pre"])
    out["dx"] = cfg["alpha"] * D
    out["D"] = D
    m = cfg["scale"] * D * keep
    n = np.where(keep > 0, _f64(b), 0.0) if cfg["post"] == "none" else _f64(b)
    if cfg["post"] != "none":
        bh = _hat(b, stats["post_mean"], stats["post_rstd"])
        n = bh * _f64(par["post_gamma"])
        if par.get("post_beta") is not None:
            n = n + _f64(par["post_beta"])
    if cfg["gate"] != "none":
        out["gate"] = (m * n).sum(axis=0 if cfg["gate"] == "channel" else 1)
    dn = m * _gate(cfg["gate"], par.get("gate"))
    if cfg["post"] == "none":
        out["db"] = dn
    else:
        out["post_gamma"], out["post_beta"] = (dn * bh).sum(axis=0), dn.sum(axis=0)
        out["db"] = _norm_bwd(b, stats["post_mean"], stats["post_rstd"], dn * _f64(par["post_gamma"]), cfg["post"])
    return out


def embedding_fwd(ids, table, scale, keep=None):
    table = _f64(table)
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < len(table))
    y = np.where(ok[:, None], scale * table[np.where(ok, ids, 0)], 0.0)
    return y if keep is None else y * keep


def embedding_bwd(ids, dy, V, scale, keep=None):
    dy = _f64(dy) if keep is None else drop(dy, keep)
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < V)
    out = np.zeros((V, dy.shape[1]))
    np.add.at(out, ids[ok], scale * dy[ok])
    return out


def layer_with_ends(x, dy, p, hq, hkv, d, ends, keep1, keep2, eps=1e-5):
    """Forward and backward of the layer with block ends, unchunked, batch 1.
    ends: norm, gate (bool), alpha, scale.  p: the layer's parameters and
    g_end1, b_end1, gate1, g_end2, b_end2, gate2 where ends has them.  keep1,
    keep2: the two dropouts' factors [S, H].  Returns y, dx and the gradients
    by the parameters' names with a d in front (dw_*, dg1, ...)."""
    x, dy = _f64(x), _f64(dy)
    S = len(x)
    cfg = [dict(post=ends["norm"], pre=pre, gate="channel" if ends["gate"] else "none", eps=eps, alpha=ends["alpha"],
                scale=ends["scale"]) for pre in ("layer", "none")]
    par = [dict(post_gamma=p.get(f"g_end{n}"), post_beta=p.get(f"b_end{n}"), gate=p.get(f"gate{n}"),
                pre_gamma=p["g2"], pre_beta=p["b2"]) for n in (1, 2)]
    w = {k: _f64(p[k]) for k in ("w_qkv", "w_o", "w_1", "w_2")}
    u, m1, r1 = layer_norm(x, p["g1"], p["b1"], eps)
    qkv = u @ w["w_qkv"]
    split = np.split(qkv, [hq * d, (hq + hkv) * d], axis=1)
    q, k, v = (t.reshape(1, S, n, d) for t, n in zip(split, (hq, hkv, hkv)))
    scale = 1.0 / math.sqrt(d)
    o4, lse = attention_fwd(q, k, v, scale)
    o = o4.reshape(S, -1)
    e1 = o @ w["w_o"]
    f1 = block_norm_fwd(x, e1, cfg[0], par[0], keep1)
    a = f1["z"] @ w["w_1"]
    g = gelu(a)
    e2 = g @ w["w_2"]
    f2 = block_norm_fwd(f1["h"], e2, cfg[1], par[1], keep2)
    out = {"y": f2["h"]}
    b2 = block_norm_bwd(e2, None, f2, None, dy, cfg[1], par[1], keep2)
    out["dw_2"] = g.T @ b2["db"]
    da = (b2["db"] @ w["w_2"].T) * gelu_grad(a)
    out["dw_1"] = f1["z"].T @ da
    b1 = block_norm_bwd(e1, f1["h"], f1, da @ w["w_1"].T, b2["dx"], cfg[0], par[0], keep1)
    out["dg2"], out["db2"] = b1["pre_gamma"], b1["pre_beta"]
    out["dw_o"] = o.T @ b1["db"]
    do4 = (b1["db"] @ w["w_o"].T).reshape(1, S, hq, d)
    dqkv = np.concatenate([t.reshape(S, -1) for t in attention_bwd(q, k, v, do4, scale, o4, lse)], axis=1)
    out["dw_qkv"] = u.T @ dqkv
    dx, out["dg1"], out["db1"] = layer_norm_bwd(x, p["g1"], m1, r1, dqkv @ w["w_qkv"].T)
    out["dx"] = b1["dx"] + dx
    for n, b in ((1, b1), (2, b2)):
        for ours, theirs in (("post_gamma", f"g_end{n}"), ("post_beta", f"b_end{n}"), ("gate", f"gate{n}")):
            if p.get(theirs) is not None:
                out["d" + theirs] = b[ours]
    return out
