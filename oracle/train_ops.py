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

Pins (tests/test_train_ops_cpu.py): the generator's published answers; the
drawn share of kept elements; central differences of every gradient; the
lookup's gradient as the transpose of the lookup.
"""
from __future__ import annotations

import numpy as np

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
    D = np.zeros_like(keep) if dh is None else _f64(dh)
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
