"""fp64 oracle of the operators that close a training step: rotary positions,
cross-entropy with its gradient, the gradient norm, and AdamW with states in 32
or in 8 bits.

TEST INFRASTRUCTURE ONLY -- never imported by the product path.

Pins (tests/test_step_ops_cpu.py): rotations keep lengths and depend on the
difference of positions alone; the loss against a loop over classes, its
gradient by central differences; the layer's gradients by central differences
of its mean loss; AdamW against a scalar loop; the 8-bit format
against a table of its codes, its rounding by its mean over the draws.
"""
from __future__ import annotations

import math

import numpy as np

from .causal_attention import attention_bwd, attention_fwd
from .train_ops import block_norm_bwd, block_norm_fwd, philox4x32
from .transformer_layer import gelu, gelu_grad, layer_norm, layer_norm_bwd


def _f64(x):
    return np.asarray(x, dtype=np.float64)


# ------------------------------------------------------------------- rotary
PI = np.longdouble("3.14159265358979323846264338327950288")


def rope_freqs(rot, base=10000.0, kind="none", factor=1.0, original_len=0.0, beta_fast=32.0, beta_slow=1.0):
    """Angles per position [rot / 2] (long double) and the amplitude."""
    ld = np.longdouble
    j, s = np.arange(rot // 2, dtype=ld), ld(factor)
    b = ld(base) * s ** (ld(rot) / (rot - 2)) if kind == "ntk" else ld(base)
    f = b ** (-2 * j / rot)
    if kind == "linear":
        f = f / s
    if kind == "yarn":
        turns = original_len * f / (2 * PI)
        c = np.clip((turns - beta_slow) / ld(beta_fast - beta_slow), 0, 1)
        f = c * f + (1 - c) * f / s
    return f, 0.1 * math.log(factor) + 1.0 if kind == "yarn" else 1.0


def rotary(x, pos, freqs, rot, layout, amp=1.0, inverse=False):
    """x [rows, heads, D] turned at positions pos [rows]; freqs as rope_freqs
    gives them, or integers: fractions of a turn in units of 2^-64."""
    x = _f64(x).copy()
    if isinstance(freqs[0], (int, np.uint64)):
        turns = np.array([[(int(p) * int(f)) % 2 ** 64 / 2.0 ** 64 for f in freqs] for p in pos])
    else:
        t = np.asarray(pos).astype(np.longdouble)[:, None] * (freqs / (2 * PI))
        turns = (t - np.floor(t)).astype(np.float64)
    w = 2 * math.pi * turns * (-1.0 if inverse else 1.0)
    c, s = amp * np.cos(w)[:, None, :], amp * np.sin(w)[:, None, :]
    i = np.arange(rot // 2)
    ia, ib = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    a, b = x[..., ia].copy(), x[..., ib].copy()
    x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
    return x


# --------------------------------------------------------------------- loss
def cross_entropy(x, t, smooth=0.0, z=0.0, scale=1.0, lse=None, dloss=None):
    """loss, lse [rows] and dx of rows of logits; zeros where t is outside.  With
    lse (and a factor dloss a row) the gradient from that lse."""
    x, t = _f64(x), np.asarray(t).astype(np.int64)
    rows, V = x.shape
    ok = (t >= 0) & (t < V)
    with np.errstate(all="ignore"):
        m = x.max(axis=1, initial=-np.inf)
        b = np.where(np.isfinite(m), m, 0.0)
        if lse is None:  # b + part: differences from b first, where b is large
            part = np.log(np.exp(x - b[:, None]).sum(axis=1))
        else:
            b, part = _f64(lse), np.zeros(rows)
        lse = b + part
        q = np.full((rows, V), smooth / V)
        q[np.arange(rows)[ok], t[ok]] += 1.0 - smooth
        loss = part + np.where(q > 0, q * (b[:, None] - x), 0.0).sum(axis=1) + (z * lse ** 2 if z else 0.0)
        w = scale * (np.ones(rows) if dloss is None else _f64(dloss))
        p = np.exp((x - b[:, None]) - part[:, None])
        dx = w[:, None] * ((1.0 + (2.0 * z * lse[:, None] if z else 0.0)) * p - q)
    return np.where(ok, loss, 0.0), np.where(ok, lse, 0.0), np.where(ok[:, None], dx, 0.0)


# ------------------------------------------------------------------- update
def grad_norm(grads, max_norm):
    n = math.sqrt(math.fsum(float(v) for g in grads for v in np.square(_f64(g)).ravel()))
    return n, min(1.0, max_norm / n) if n > 0 else 1.0


def adamw(p, g, m, v, t, lr, b1, b2, eps, wd, f=1.0):
    """New p, m, v."""
    g = f * _f64(g)
    m = b1 * _f64(m) + (1.0 - b1) * g
    v = b2 * _f64(v) + (1.0 - b2) * g * g
    with np.errstate(invalid="ignore", divide="ignore"):
        q = (m / (1.0 - b1 ** t)) / (np.sqrt(v / (1.0 - b2 ** t)) + eps)
    return _f64(p) - lr * (q + wd * _f64(p)), m, v


# The 127 finite magnitudes of e4m3 by code: 3 bits of mantissa, exponent bias 7.
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def value8(codes, scales):
    """Values of e4m3 codes [n] under exponent bytes [ceil(n / 32)]."""
    codes = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    mag = np.append(E4M3, np.nan)[codes & 127]
    k = np.repeat(np.asarray(scales, dtype=np.int64), 32)[:len(codes)]
    return np.where(codes >= 128, -1.0, 1.0) * mag * np.where(k > 0, 2.0 ** (k - 127.0), 0.0)


def block_bytes(x):
    """The exponent byte of each block of 32."""
    x = np.abs(_f64(x))
    x = np.where(np.isfinite(x), x, 0.0)
    out = []
    for b in range(0, len(x), 32):
        a, k = x[b:b + 32].max(), 1
        if a > 0:
            k = max(1, int(math.floor(math.log2(a))) - 8 + 127 - 2)
            while a > 448.0 * 2.0 ** (k - 127):
                k += 1
        out.append(k)
    return np.array(out, dtype=np.uint8)


def draws(n, block0, t, seed):
    """The 32-bit words of a tensor's n elements: low half m's, high half r's."""
    g = np.arange(-(-n // 4), dtype=np.uint64) + np.uint64(8 * block0)
    u32 = np.uint64(0xFFFFFFFF)
    ctr = np.stack([g & u32, g >> np.uint64(32), np.full_like(g, t & 0xFFFFFFFF), np.full_like(g, t >> 32)], axis=-1)
    return philox4x32(ctr, (seed & 0xFFFFFFFF, seed >> 32)).reshape(-1)[:n]


def round8(x, scales, u, positive):
    """x to e4m3 codes: down, or up where the share of the step that is cut off
    and u / 65536 make one.  Returns (codes, values, distance of the draw's
    threshold from the share, in steps)."""
    x = _f64(x)
    unit = 2.0 ** (np.repeat(scales.astype(np.float64), 32)[:len(x)] - 127)
    y = np.abs(x) / unit
    bad = ~np.isfinite(y)
    y = np.where(bad, 0.0, y)
    lo = np.searchsorted(E4M3, y, side="right") - 1
    step = np.where(lo < 126, E4M3[np.minimum(lo + 1, 126)] - E4M3[lo], 32.0)
    share = (y - E4M3[lo]) / step + u / 65536.0
    code = np.minimum(lo + (share >= 1.0), 126)
    if positive:
        code = np.where((x > 0) & (code == 0), 1, code)
    code = np.where(bad, 127, code)
    sign = np.where(np.signbit(x), 128, 0)
    return (code + sign).astype(np.uint8), np.abs(share - 1.0)


# -------------------------------------------------------------------- the layer
def layer_step(x, p, hq, hkv, d, rope, targets, smooth=0.0, z=0.0, scale=1.0, ends=None, keep=(1.0, 1.0), eps=1e-5):
    """A layer's forward and backward with rotary positions (rope: rot, layout,
    freqs, amp, position0) and the loss of its output, unchunked, batch 1.
    ends: as layer_with_ends takes them (None: plain adds).  Returns y, loss, dx
    and the parameters' gradients by their names with a d in front."""
    x = _f64(x)
    S = len(x)
    w = {k: _f64(v) for k, v in p.items()}
    ends = ends or dict(norm="none", gate=False, alpha=1.0, scale=1.0)
    cfg = [dict(post=ends["norm"], pre=pre, gate="channel" if ends["gate"] else "none", eps=eps, alpha=ends["alpha"],
                scale=ends["scale"]) for pre in ("layer", "none")]
    par = [dict(post_gamma=w.get(f"g_end{n}"), post_beta=w.get(f"b_end{n}"), gate=w.get(f"gate{n}"),
                pre_gamma=w["g2"], pre_beta=w["b2"]) for n in (1, 2)]
    keep = [np.ones(x.shape) * k for k in keep]
    pos = np.arange(S) + rope["position0"]
    how = (rope["freqs"], rope["rot"], rope["layout"], rope["amp"])
    turn = lambda t, inv: rotary(t[0], pos, *how, inv)[None]  # noqa: E731
    u, m1, r1 = layer_norm(x, w["g1"], w["b1"], eps)
    split = np.split(u @ w["w_qkv"], [hq * d, (hq + hkv) * d], axis=1)
    q, k, v = (t.reshape(1, S, n, d) for t, n in zip(split, (hq, hkv, hkv)))
    q, k = turn(q, False), turn(k, False)
    sm = 1.0 / math.sqrt(d)
    o4, lse = attention_fwd(q, k, v, sm)
    o = o4.reshape(S, -1)
    e1 = o @ w["w_o"]
    f1 = block_norm_fwd(x, e1, cfg[0], par[0], keep[0])
    a = f1["z"] @ w["w_1"]
    g = gelu(a)
    e2 = g @ w["w_2"]
    f2 = block_norm_fwd(f1["h"], e2, cfg[1], par[1], keep[1])
    y = f2["h"]
    uf, mf, rf = layer_norm(y, w["gf"], w["bf"], eps)
    loss, _, dl = cross_entropy(uf @ w["w_out"], targets, smooth, z, scale)
    out = {"y": y, "loss": loss, "dw_out": uf.T @ dl}
    dy, out["dgf"], out["dbf"] = layer_norm_bwd(y, w["gf"], mf, rf, dl @ w["w_out"].T)
    b2 = block_norm_bwd(e2, None, f2, None, dy, cfg[1], par[1], keep[1])
    out["dw_2"] = g.T @ b2["db"]
    da = (b2["db"] @ w["w_2"].T) * gelu_grad(a)
    out["dw_1"] = f1["z"].T @ da
    b1 = block_norm_bwd(e1, f1["h"], f1, da @ w["w_1"].T, b2["dx"], cfg[0], par[0], keep[0])
    out["dg2"], out["db2"] = b1["pre_gamma"], b1["pre_beta"]
    out["dw_o"] = o.T @ b1["db"]
    dq, dk, dv = attention_bwd(q, k, v, (b1["db"] @ w["w_o"].T).reshape(1, S, hq, d), sm, o4, lse)
    dqkv = np.concatenate([t.reshape(S, -1) for t in (turn(dq, True), turn(dk, True), dv)], axis=1)
    out["dw_qkv"] = u.T @ dqkv
    dx, out["dg1"], out["db1"] = layer_norm_bwd(x, w["g1"], m1, r1, dqkv @ w["w_qkv"].T)
    out["dx"] = b1["dx"] + dx
    for n, b in ((1, b1), (2, b2)):
        for ours, theirs in (("post_gamma", f"g_end{n}"), ("post_beta", f"b_end{n}"), ("gate", f"gate{n}")):
            if theirs in p:
                out["d" + theirs] = b[ours]
    return out
