"""The training operators on the GPU against the fp64 oracle: dropout, the
norms, gate and residual at a block's end, the embedding and its gradient.

Tolerances count roundings.  u = 2^-24 is half a step of fp32, half(t) that of
the output's type (bf16 2^-8, fp32 2^-24), relative to the value.  A sum of
terms added over a depth of d additions is off by at most d u times the sum
of the terms' magnitudes; each test names its depth.
"""
import sys

import numpy as np
import pytest
import torch

from oracle import train_ops as O
from paper_2503_10377_amd import sppo as L
from parity import to_np

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF, "f32": F32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


def announce(msg):
    print(f"\n[case] {msg}", file=sys.stderr, flush=True)


def randn(rows, W, ld, dtype, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, ld, generator=g) * scale + shift).to(DT[dtype])


def within(got, ref, tol, what):
    """|got - ref| <= tol, element by element (NaN and infinities alike)."""
    got, ref = to_np(got), np.asarray(ref)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= tol))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(),
                           got[bad][:3], ref[bad][:3], np.broadcast_to(tol, ref.shape)[bad][:3])


# ------------------------------------------------------------------ dropout
def drop_tol(x, keep, res, dtype):
    """The scale, the product and the sum round once each in fp32, then the
    output's type."""
    v = O.drop(x, keep)
    ref = v + (0.0 if res is None else to_np(res))
    mag = np.abs(v) + (0.0 if res is None else np.abs(to_np(res)))
    return ref, HALF[dtype] * np.abs(ref) + 4 * U * mag


@pytest.mark.parametrize("rows,W,ld,dtype,res,p,row0", [
    (1, 8, 8, "bf16", False, 0.5, 0),
    (1, 4096, 4096, "bf16", True, 0.1, 3),
    (33, 264, 272, "bf16", True, 0.3, 2 ** 33),          # strided, element indices past 32 bits
    (257, 1024, 1024, "f32", False, 0.1, 7),
    (65, 8200, 8208, "f32", True, 0.75, 2 ** 40 + 1),
    (2051, 40, 40, "bf16", False, 0.01, 0),
    (5, 64, 64, "bf16", True, 0.0, 0),                   # nothing dropped
    (5, 64, 64, "f32", False, 0.99998, 0),               # all but the highest draw dropped (T = 65535)
    (4100, 4096, 4104, "bf16", True, 0.1, 0),            # read past the caches, strided and dense
    (1030, 8192, 8192, "f32", False, 0.1, 0),
])
def test_dropout(rows, W, ld, dtype, res, p, row0):
    announce(f"dropout rows={rows} W={W} ld={ld} {dtype} res={res} p={p} row0={row0}")
    x = randn(rows, W, ld, dtype, 1)
    r = randn(rows, W, ld, dtype, 2) if res else None
    seed, offset = 0xFEDCBA9876543210, 2 ** 40 + 17
    y = torch.full((rows, ld), 7.0, device="cuda", dtype=DT[dtype])
    L.sppo_dropout(rows, W, x.cuda(), ld, L.drop_spec(p, seed, offset, row0), y, ld, None if r is None else r.cuda(),
                   ld, dtype)
    keep = O.keep_factor(rows, W, p, seed, offset, row0)
    ref, tol = drop_tol(to_np(x)[:, :W], keep, None if r is None else r[:, :W], dtype)
    within(y[:, :W], ref, tol, "y")
    assert torch.all(y[:, W:] == 7.0), "columns past the width written"


def test_dropout_in_place_and_on_chunks():
    """y over x, y over res, and a sequence in ragged chunks: the same bits."""
    rows, W, p, seed, off = 300, 512, 0.2, 11, 5
    announce("dropout in place, chunks")
    x, r = randn(rows, W, W, "bf16", 3).cuda(), randn(rows, W, W, "bf16", 4).cuda()
    whole = torch.empty_like(x)
    L.sppo_dropout(rows, W, x, W, L.drop_spec(p, seed, off, 50), whole, W, r, W)
    a, b = x.clone(), r.clone()
    L.sppo_dropout(rows, W, a, W, L.drop_spec(p, seed, off, 50), a, W, r, W)
    L.sppo_dropout(rows, W, x, W, L.drop_spec(p, seed, off, 50), b, W, b, W)
    parts = torch.empty_like(x)
    for c0, c1 in ((0, 1), (1, 130), (130, 300)):
        L.sppo_dropout(c1 - c0, W, x[c0:], W, L.drop_spec(p, seed, off, 50 + c0), parts[c0:], W, r[c0:], W)
    for t in (a, b, parts):
        assert torch.equal(t, whole)


def test_dropout_masks_what_it_drops():
    """NaN and infinities at dropped places are gone, at kept ones they stay."""
    rows, W = 16, 256
    announce("dropout of NaN and infinities")
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.full((rows, W), bad, device="cuda", dtype=BF)
        y = torch.empty_like(x)
        L.sppo_dropout(rows, W, x, W, L.drop_spec(0.5, 9), y, W)
        within(y, np.where(O.keep_factor(rows, W, 0.5, 9) > 0, bad, 0.0), 0.0, bad)


def test_dropout_past_a_launch():
    """More elements than one launch takes (2^33), in place; rows at both ends
    and around the boundary."""
    W = 16384
    rows = 2 ** 33 // W + 3
    announce(f"dropout rows={rows} W={W}")
    x = torch.ones(rows, W, device="cuda", dtype=BF)
    L.sppo_dropout(rows, W, x, W, L.drop_spec(0.25, 13, 1), x, W)
    for r in (0, 1, rows // 2, rows - 4, rows - 3, rows - 2, rows - 1):
        keep = O.keep_factor(1, W, 0.25, 13, 1, row0=r)
        within(x[r:r + 1], keep, HALF["bf16"] * keep, r)


def test_dropout_replayed_in_a_graph_draws_new_masks():
    """A captured call adds a device counter to its offset: every replay has
    the mask of the counter's value at that time, as an eager call with it."""
    rows, W, p = 64, 1024, 0.3
    announce("dropout in a graph")
    x = randn(rows, W, W, "bf16", 6).cuda()
    y = torch.empty_like(x)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    spec = L.drop_spec(p, 21, 100, 0, step)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        L.sppo_dropout(rows, W, x, W, spec, y, W)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        L.sppo_dropout(rows, W, x, W, spec, y, W)
    for i in (0, 1, 5, 2 ** 33):
        step.fill_(i)
        y.zero_()
        graph.replay()
        eager = torch.empty_like(x)
        L.sppo_dropout(rows, W, x, W, L.drop_spec(p, 21, 100 + i), eager, W)
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i
        ref, tol = drop_tol(to_np(x), O.keep_factor(rows, W, p, 21, 100 + i), None, "bf16")
        within(y, ref, tol, i)


# ------------------------------------------------------------------ block norm
class Case:
    """Inputs of one block end, on the host and the device."""

    def __init__(self, rows, H, ld, dtype, post, pre, gate, beta=True, p=0.0, alpha=1.0, scale=1.0, seed=0, row0=0,
                 eps=1e-5):
        self.rows, self.H, self.ld, self.dtype, self.p, self.row0 = rows, H, ld, dtype, p, row0
        self.cfg = dict(post=post, pre=pre, gate=gate, eps=eps, alpha=float(np.float32(alpha)),
                        scale=float(np.float32(scale)))
        self.cfg["eps"] = float(np.float32(eps))
        g = torch.Generator().manual_seed(100 + seed)
        self.x = randn(rows, H, ld, dtype, seed + 1, 2.0, 0.25)
        self.b = randn(rows, H, ld, dtype, seed + 2, 1.5, -0.5)
        self.par = {}
        for k, kind in (("post", post), ("pre", pre)):
            if kind != "none":
                self.par[k + "_gamma"] = 1 + 0.2 * torch.randn(H, generator=g)
                if beta:
                    self.par[k + "_beta"] = 0.3 * torch.randn(H, generator=g)
        if gate != "none":
            self.par["gate"] = 0.5 + torch.rand(H if gate == "channel" else rows, generator=g)
        self.dpar = {k: v.cuda() for k, v in self.par.items()}
        self.npar = {k: to_np(v) for k, v in self.par.items()}
        self.seed, self.offset = 0x123456789ABCDEF0 + seed, 3
        self.drop = L.drop_spec(p, self.seed, self.offset, row0) if p > 0 else None
        self.keep = O.keep_factor(rows, H, p, self.seed, self.offset, row0) if p > 0 else np.ones((rows, H))
        self.bn = L.block_norm(H, dtype, post, pre, gate, eps, alpha, scale, **self.dpar)
        self.stats = {}
        for k, kind in (("post", post), ("pre", pre)):
            if kind == "layer":
                self.stats[k + "_mean"] = torch.full((rows,), float("nan"), device="cuda")
            if kind != "none":
                self.stats[k + "_rstd"] = torch.full((rows,), float("nan"), device="cuda")
        self.cstats = L.block_norm_stats(**self.stats)

    def act(self, fill=7.0):
        return torch.full((self.rows, self.ld), fill, device="cuda", dtype=DT[self.dtype])

    def forward(self, stream=None):
        h, z = self.act(), self.act() if self.cfg["pre"] != "none" else None
        ld = self.ld
        L.sppo_block_norm_fwd(self.bn, self.rows, self.drop, self.x.cuda(), ld, self.b.cuda(), ld, h, ld, z, ld,
                              self.cstats, stream)
        return h, z

    def np_stats(self):
        z = np.zeros(self.rows)
        return {k: to_np(self.stats[k]) if k in self.stats else z
                for k in ("post_mean", "post_rstd", "pre_mean", "pre_rstd")}


def rowmean(a):
    return a.mean(axis=1, keepdims=True)


def norm_error(v, e, kind, mean, rstd):
    """Bounds of the errors of the mean, the relative error of 1/std and the
    error of the normalised value, for a row known up to e: sums of at most
    1024 columns a wave are 8 to 16 additions a thread and 6 across the wave,
    then up to 16 waves: a depth below 40; squares and their sum another 40,
    half of it (and 4 roundings) in 1/std; d = v - mean and d rstd round too."""
    mean, rstd = mean[:, None], rstd[:, None]
    em = rowmean(e) + 40 * U * rowmean(np.abs(v)) if kind == "layer" else 0.0 * rowmean(e)
    d = np.abs(v - mean)
    # var's relative error: 2 mean(|d| e_d) rstd^2 from the values, 44 u from the sums
    er = rstd ** 2 * rowmean(d * (e + em)) + 30 * U
    ed = e + em + U * d
    return em, er, ed * rstd + d * rstd * (er + 2 * U)


def fwd_check(c, h, z):
    cfg, par = c.cfg, c.npar
    x, b = to_np(c.x)[:, :c.H], to_np(c.b)[:, :c.H]
    ref = O.block_norm_fwd(x, b, cfg, par, c.keep)
    n, en = b, np.zeros_like(b)
    if cfg["post"] != "none":
        m, r = ref["post_mean"], ref["post_rstd"]
        em, er, eh = norm_error(b, en, cfg["post"], m, r)
        bh, g, bt = (b - m[:, None]) * r[:, None], np.abs(par["post_gamma"]), np.abs(par.get("post_beta", np.zeros(c.H)))
        n = bh * par["post_gamma"] + par.get("post_beta", 0.0)
        en = g * eh + 2 * U * (g * np.abs(bh) + bt)
        if cfg["post"] == "layer":
            within(c.stats["post_mean"], m, em[:, 0], "post_mean")
        within(c.stats["post_rstd"], r, r * er[:, 0], "post_rstd")
    gate = {"none": 1.0, "channel": par.get("gate", 0), "token": np.reshape(par.get("gate", 0), (-1, 1))}[cfg["gate"]]
    k = np.abs(gate * c.keep * cfg["scale"])
    branch = k * np.abs(n)
    eh = k * en + 6 * U * branch + 2 * U * (np.abs(cfg["alpha"] * x) + branch)
    within(h[:, :c.H], ref["h"], HALF[c.dtype] * np.abs(ref["h"]) * (1 + 1e-3) + (1 + HALF[c.dtype]) * eh, "h")
    assert torch.all(h[:, c.H:] == 7.0)
    if z is None:
        return
    m, r = ref["pre_mean"], ref["pre_rstd"]
    em, er, ez = norm_error(ref["h"], eh, cfg["pre"], m, r)
    hh = (ref["h"] - m[:, None]) * r[:, None]
    ez = np.abs(par["pre_gamma"]) * ez + 2 * U * (np.abs(hh * par["pre_gamma"]) + np.abs(par.get("pre_beta", 0.0)))
    if cfg["pre"] == "layer":
        within(c.stats["pre_mean"], m, em[:, 0], "pre_mean")
    within(c.stats["pre_rstd"], r, r * er[:, 0], "pre_rstd")
    within(z[:, :c.H], ref["z"], HALF[c.dtype] * np.abs(ref["z"]) + (1 + HALF[c.dtype]) * ez, "z")
    assert torch.all(z[:, c.H:] == 7.0)


def back_error(v, e_v, g, e_g, kind, mean, rstd):
    """Gradient at a norm's input from g at the normalised value, and its
    error where g is known up to e_g: the two means over the row are sums of
    depth below 40 of products of 3 factors; 8 more roundings put the value
    together.  (The statistics are the call's inputs, exact.)"""
    vh = np.abs(v - mean[:, None]) * rstd[:, None]
    vm = (np.abs(v) + np.abs(mean[:, None])) * rstd[:, None]  # what the rounding of v - mean is relative to
    m1 = rowmean(np.abs(g)) if kind == "layer" else 0.0
    e1 = rowmean(e_g) + 44 * U * m1 if kind == "layer" else 0.0
    m2 = rowmean(np.abs(g) * vh)
    e2 = rowmean(e_g * vh) + 48 * U * rowmean(np.abs(g) * vm)
    return rstd[:, None] * (e_g + e1 + vh * e2 + 8 * U * (np.abs(g) + m1 + vm * m2)), vm


def run_bwd(c, h, dz, dh, acc=0, grads=None, ws=None, stream=None):
    ld, H = c.ld, c.H
    dx, db = c.act(), c.act()
    g = {k: torch.full_like(v, 0.5) for k, v in c.dpar.items()} if grads is None else grads
    nb = L.sppo_block_norm_bwd_workspace(c.bn, c.rows)
    ws = torch.full((max(nb // 4, 4),), float("nan"), device="cuda") if ws is None else ws
    L.sppo_block_norm_bwd(c.bn, c.rows, c.drop, c.b.cuda(), ld, h, ld, c.cstats, dz, ld, dh, ld, dx, ld, db, ld,
                          L.block_norm_grads(**g), ws, nb, acc, stream)
    return dx, db, g


def bwd_check(c, h, dz, dh, dx, db, g, start=0.0):
    cfg, par, H = c.cfg, c.npar, c.H
    b, hn = to_np(c.b)[:, :H], to_np(h)[:, :H]
    dzn = None if dz is None else to_np(dz)[:, :H]
    dhn = None if dh is None else to_np(dh)[:, :H]
    st = c.np_stats()
    ref = O.block_norm_bwd(b, hn, st, dzn, dhn, cfg, par, c.keep)
    D = ref["D"]
    eD = np.zeros_like(D)
    # Column sums: a team adds its rows one by one (a workgroup has at most
    # ceil(rows / 256) + 8 of them), then a workgroup's up to 8 teams, then up
    # to 512 workgroups' in 32 groups of 16 and a tree of 5.
    depth = -(-c.rows // 256) + 8 + 8 + 16 + 5 + 4

    def col(name, terms, err, axis=0):
        if name in g:
            tol = err.sum(axis=axis) + depth * U * np.abs(terms).sum(axis=axis)
            within(g[name], ref[name] + start, tol + 2 * U * (np.abs(ref[name]) + abs(start)), name)

    if cfg["pre"] != "none":
        gz = dzn * par["pre_gamma"]
        eD, vm = back_error(hn, 0, gz, U * np.abs(gz), cfg["pre"], st["pre_mean"], st["pre_rstd"])
        col("pre_gamma", dzn * vm, 3 * U * np.abs(dzn) * vm)
        col("pre_beta", dzn, 0 * dzn)
    eD = eD + 2 * U * (np.abs(D) + (0 if dhn is None else np.abs(dhn)))
    a = abs(cfg["alpha"])
    within(dx[:, :H], ref["dx"], HALF[c.dtype] * np.abs(ref["dx"]) + (1 + HALF[c.dtype]) * (a * eD + U * a * np.abs(D)),
           "dx")
    s = abs(cfg["scale"]) * c.keep
    m, em = s * np.abs(D), s * eD + 4 * U * s * np.abs(D)
    gate = {"none": np.ones((1, 1)), "channel": np.reshape(par.get("gate", 0), (1, -1)),
            "token": np.reshape(par.get("gate", 0), (-1, 1))}[cfg["gate"]]
    tok = gate if cfg["gate"] == "token" else 1.0
    if cfg["post"] == "none":
        dn, en = gate * m, gate * em + 2 * U * gate * m
        within(db[:, :H], ref["db"], HALF[c.dtype] * np.abs(ref["db"]) + (1 + HALF[c.dtype]) * en, "db")
        if cfg["gate"] == "channel":
            col("gate", m * np.abs(b), em * np.abs(b) + 2 * U * m * np.abs(b))
        elif cfg["gate"] == "token" and "gate" in g:
            e = (em * np.abs(b)).sum(axis=1) + 44 * U * (m * np.abs(b)).sum(axis=1)
            within(g["gate"], ref["gate"], e, "gate")
    else:
        gm, bt = np.abs(par["post_gamma"]), np.abs(par.get("post_beta", np.zeros(H)))
        w, ew = gate * m * gm, gate * em * gm + 3 * U * gate * m * gm
        e, vm = back_error(b, 0, w, ew, cfg["post"], st["post_mean"], st["post_rstd"])
        within(db[:, :H], ref["db"], HALF[c.dtype] * np.abs(ref["db"]) + (1 + HALF[c.dtype]) * e, "db")
        # gamma, beta and a channel's gate: from sums of (token gate) m bh and (token gate) m
        cg = gate if cfg["gate"] == "channel" else 1.0
        t2, e2 = tok * m * vm, tok * em * vm + 5 * U * tok * m * vm
        t3, e3 = tok * m, tok * em + 2 * U * tok * m
        col("post_gamma", cg * t2, cg * e2)
        col("post_beta", cg * t3, cg * e3)
        if cfg["gate"] == "channel":
            col("gate", gm * t2 + bt * t3, gm * e2 + bt * e3)
        elif cfg["gate"] == "token" and "gate" in g:
            t = m * (gm * vm + bt)
            e = (em * (gm * vm + bt)).sum(axis=1) + 50 * U * t.sum(axis=1)
            within(g["gate"], ref["gate"], e, "gate")
    for t in (dx, db):
        assert torch.all(t[:, H:] == 7.0), "columns past H written"


NORM_CASES = [
    # rows, H, ld, dtype, post, pre, gate, beta, p, alpha, scale
    (1, 8, 8, "bf16", "layer", "layer", "channel", True, 0.5, 1.0, 1.0),
    (1, 4096, 4096, "bf16", "layer", "layer", "channel", True, 0.1, 1.0, 0.5),
    (3, 512, 520, "f32", "rms", "rms", "token", False, 0.2, 0.9, 1.0),
    (37, 264, 264, "bf16", "none", "layer", "none", True, 0.1, 1.0, 1.0),
    (130, 520, 528, "bf16", "layer", "none", "token", True, 0.0, 1.0, 0.25),
    (65, 1024, 1024, "f32", "none", "rms", "channel", True, 0.3, 1.2, 1.0),
    (33, 1032, 1040, "bf16", "rms", "layer", "channel", False, 0.0, 1.0, 1.0),
    (70, 2056, 2056, "f32", "layer", "rms", "token", True, 0.1, -0.5, 2.0),
    (600, 2048, 2048, "bf16", "rms", "rms", "none", False, 0.1, 1.0, 1.0),
    (19, 4104, 4112, "bf16", "layer", "layer", "token", True, 0.1, 1.0, 1.0),
    (40, 8192, 8192, "f32", "layer", "layer", "channel", True, 0.1, 1.0, 1.0),
    (2, 8192, 8200, "bf16", "none", "none", "channel", False, 0.4, 1.0, 1.0),
    (5000, 72, 72, "bf16", "layer", "layer", "channel", True, 0.1, 1.0, 1.0),
    (9, 64, 64, "f32", "none", "none", "none", False, 0.0, 0.0, 1.0),
    (1000, 128, 136, "f32", "rms", "layer", "token", True, 0.1, 1.0, 1.0),
    (77, 136, 136, "bf16", "layer", "rms", "channel", True, 0.1, 1.0, 1.0),
    (33, 256, 256, "f32", "none", "layer", "channel", True, 0.1, 1.0, 1.0),
    (1100, 768, 768, "bf16", "layer", "layer", "channel", True, 0.1, 1.0, 1.0),
    (515, 3000, 3008, "bf16", "layer", "layer", "channel", True, 0.1, 1.0, 1.0),
    (4100, 4096, 4104, "bf16", "layer", "layer", "channel", True, 0.1, 1.0, 1.0),  # read past the caches
]


@pytest.mark.parametrize("rows,H,ld,dtype,post,pre,gate,beta,p,alpha,scale", NORM_CASES)
def test_block_norm(rows, H, ld, dtype, post, pre, gate, beta, p, alpha, scale):
    announce(f"block norm rows={rows} H={H} ld={ld} {dtype} post={post} pre={pre} gate={gate} p={p}")
    c = Case(rows, H, ld, dtype, post, pre, gate, beta, p, alpha, scale, seed=rows + H, row0=12345)
    h, z = c.forward()
    fwd_check(c, h, z)
    dz = randn(rows, H, ld, dtype, 50).cuda() if pre != "none" else None
    dh = randn(rows, H, ld, dtype, 51).cuda()
    dx, db, g = run_bwd(c, h, dz, dh)
    bwd_check(c, h, dz, dh, dx, db, g)
    # added to, and the same bits again
    dx2, db2, g2 = run_bwd(c, h, dz, dh, acc=1)
    bwd_check(c, h, dz, dh, dx2, db2, {k: v for k, v in g2.items() if not (k == "gate" and gate == "token")}, start=0.5)
    dx3, db3, g3 = run_bwd(c, h, dz, dh)
    assert torch.equal(dx, dx3) and torch.equal(db, db3) and torch.equal(dx, dx2) and torch.equal(db, db2)
    for k in g:
        assert torch.equal(g[k], g3[k]), k
    if gate == "token":
        assert torch.equal(g["gate"], g2["gate"])


@pytest.mark.parametrize("dtype,H", [("bf16", H) for H in (128, 256, 512, 1024, 1536, 2048, 2560, 5120, 8192)] +
                         [("f32", H) for H in (128, 256, 512, 1024, 2048, 2560, 4096, 8192)])
@pytest.mark.parametrize("post,gate", [("layer", "channel"), ("none", "token"), ("none", "none")])
def test_block_norm_of_large_activations(dtype, H, post, gate):
    """Activations of 32 MiB and more are read past the caches: the same bits
    per row as the same rows in three smaller calls have."""
    rows = 2 ** 25 // (H * DT[dtype].itemsize) + 3
    announce(f"large block norm rows={rows} H={H} {dtype} post={post} gate={gate}")
    g = torch.Generator(device="cuda").manual_seed(H)
    x, b, dz, dh = (torch.randn(rows, H, generator=g, device="cuda").to(DT[dtype]) for _ in range(4))
    par = {k: 0.5 + torch.rand(H, generator=g, device="cuda") for k in
           ["pre_gamma", "pre_beta"] + (["post_gamma", "post_beta"] if post != "none" else [])}
    token = 0.5 + torch.rand(rows, generator=g, device="cuda")
    if gate == "channel":
        par["gate"] = 0.5 + torch.rand(H, generator=g, device="cuda")

    def run(c0, c1):
        n = c1 - c0
        mine = dict(par, gate=token[c0:c1]) if gate == "token" else par
        bn = L.block_norm(H, dtype, post, "layer", gate, 1e-5, 1.0, 0.5, **mine)
        names = ["pre_mean", "pre_rstd"] + (["post_mean", "post_rstd"] if post != "none" else [])
        stats = {k: torch.empty(n, device="cuda") for k in names}
        st, drop = L.block_norm_stats(**stats), L.drop_spec(0.1, 31, 2, c0)
        h, z, dx, db = (torch.empty(n, H, device="cuda", dtype=DT[dtype]) for _ in range(4))
        grads = {k: torch.empty_like(v) for k, v in mine.items()}
        L.sppo_block_norm_fwd(bn, n, drop, x[c0:c1], H, b[c0:c1], H, h, H, z, H, st)
        nb = L.sppo_block_norm_bwd_workspace(bn, n)
        ws = torch.empty(max(nb // 4, 4), device="cuda")
        L.sppo_block_norm_bwd(bn, n, drop, b[c0:c1], H, h, H, st, dz[c0:c1], H, dh[c0:c1], H, dx, H, db, H,
                              L.block_norm_grads(**grads), ws, nb, 0)
        torch.cuda.synchronize()
        return [h, z, dx, db] + list(stats.values()) + ([grads["gate"]] if gate == "token" else []), grads, stats, h

    whole, grads, stats, h = run(0, rows)
    parts = [run(c0, c1)[0] for c0, c1 in ((0, 7), (7, rows // 2), (rows // 2, rows))]
    for i, t in enumerate(whole):
        assert torch.equal(t, torch.cat([q[i] for q in parts])), i
    # the column sums, at the depth that bwd_check derives: of dz, and of dz
    # times the normalised value, which rounds twice more and the product once
    depth = -(-rows // 256) + 8 + 8 + 16 + 5 + 4
    d = dz.double()
    within(grads["pre_beta"], to_np(d.sum(0)), to_np((depth + 2) * U * d.abs().sum(0)), "pre_beta")
    m, r = stats["pre_mean"].double()[:, None], stats["pre_rstd"].double()[:, None]
    mag = d.abs() * (h.double().abs() + m.abs()) * r
    within(grads["pre_gamma"], to_np((d * (h.double() - m) * r).sum(0)), to_np((depth + 5) * U * mag.sum(0)),
           "pre_gamma")


def test_block_norm_without_dh_and_with_frozen_parameters():
    announce("block norm: no dh, some gradients not wanted")
    c = Case(50, 256, 256, "bf16", "layer", "layer", "channel", True, 0.2, seed=4)
    h, _ = c.forward()
    dz = randn(50, 256, 256, "bf16", 60).cuda()
    dx, db, g = run_bwd(c, h, dz, None)
    bwd_check(c, h, dz, None, dx, db, g)
    for keep in (("gate",), ("post_beta", "pre_gamma"), ()):
        some = {k: torch.full_like(c.dpar[k], 0.5) for k in keep}
        dx2, db2, _ = run_bwd(c, h, dz, None, grads=some)
        assert torch.equal(dx, dx2) and torch.equal(db, db2)
        for k in keep:
            assert torch.equal(some[k], g[k]), k


def test_block_norm_backward_without_the_branch():
    """No norm after the branch and no gate gradient wanted: b is not needed."""
    announce("block norm without b")
    for gate in ("channel", "token", "none"):
        c = Case(37, 520, 520, "bf16", "none", "rms", gate, True, 0.2, seed=5)
        h, _ = c.forward()
        dz, dh = randn(37, 520, 520, "bf16", 65).cuda(), randn(37, 520, 520, "bf16", 66).cuda()
        dx, db, g = run_bwd(c, h, dz, dh)
        dx2, db2, dpre = c.act(), c.act(), torch.empty_like(g["pre_gamma"])
        nb = L.sppo_block_norm_bwd_workspace(c.bn, 37)
        ws = torch.empty(nb // 4, device="cuda")
        L.sppo_block_norm_bwd(c.bn, 37, c.drop, None, 0, h, 520, c.cstats, dz, 520, dh, 520, dx2, 520, db2, 520,
                              L.block_norm_grads(pre_gamma=dpre), ws, nb, 0)
        assert torch.equal(dx, dx2) and torch.equal(db, db2) and torch.equal(dpre, g["pre_gamma"])


def test_block_norm_in_place():
    """h over x, z over b; dx over dh, db over dz: the same bits."""
    announce("block norm in place")
    for H in (256, 4096):
        c = Case(21, H, H, "bf16", "layer", "rms", "token", True, 0.1, seed=9)
        h, z = c.forward()
        x, b = c.x.cuda(), c.b.cuda()
        L.sppo_block_norm_fwd(c.bn, 21, c.drop, x, H, b, H, x, H, b, H, c.cstats)
        assert torch.equal(x, h) and torch.equal(b, z)
        dz, dh = randn(21, H, H, "bf16", 61).cuda(), randn(21, H, H, "bf16", 62).cuda()
        dx, db, g = run_bwd(c, h, dz, dh)
        nb = L.sppo_block_norm_bwd_workspace(c.bn, 21)
        ws = torch.empty(nb // 4, device="cuda")
        L.sppo_block_norm_bwd(c.bn, 21, c.drop, c.b.cuda(), H, h, H, c.cstats, dz, H, dh, H, dh, H, dz, H,
                              L.block_norm_grads(**g), ws, nb, 0)
        assert torch.equal(dh, dx) and torch.equal(dz, db)


FWD_ALIASES = [("x", None), ("b", None), ("x", "b"), (None, "b")]                    # h and z over
BWD_ALIASES = [("dh", None), ("dz", None), (None, "b"), (None, "dz"), (None, "h"),   # dx and db over
               ("dh", "b"), ("dh", "dz"), ("dh", "h"), ("dz", "b"), ("dz", "h")]


@pytest.mark.parametrize("rows,H,dtype", [
    (9000, 120, "bf16"), (9000, 200, "f32"), (5000, 512, "bf16"), (9000, 1024, "f32"), (3000, 1536, "bf16"),
    (3000, 2048, "bf16"), (2000, 2560, "f32"), (1500, 4096, "f32"), (5000, 4096, "bf16"), (900, 5120, "bf16"),
    (700, 8192, "f32"), (2100, 8192, "f32"),
])
@pytest.mark.parametrize("post,gate", [("layer", "token"), ("none", "channel"), ("none", "none")])
def test_block_norm_over_its_inputs(rows, H, dtype, post, gate):
    """Every output that may be the buffer of an input, in every layout of a
    row, with more rows than there are teams: the bits of separate buffers."""
    announce(f"block norm over its inputs rows={rows} H={H} {dtype} post={post} gate={gate}")
    g = torch.Generator(device="cuda").manual_seed(H)
    src = {k: torch.randn(rows, H, generator=g, device="cuda").to(DT[dtype]) for k in ("x", "b", "dz", "dh")}
    rand = lambda n: 0.5 + torch.rand(n, generator=g, device="cuda")  # noqa: E731
    par = {k: rand(H) for k in ["pre_gamma", "pre_beta"] + (["post_gamma", "post_beta"] if post != "none" else [])}
    if gate != "none":
        par["gate"] = rand(rows if gate == "token" else H)
    bn = L.block_norm(H, dtype, post, "layer", gate, 1e-5, 0.9, 0.5, **par)
    st = {k: torch.empty(rows, device="cuda") for k in ("post_mean", "post_rstd", "pre_mean", "pre_rstd")}
    cst, drop = L.block_norm_stats(**st), L.drop_spec(0.1, 33, 1, 70)
    nb = L.sppo_block_norm_bwd_workspace(bn, rows)
    ws = torch.empty(nb // 4, device="cuda")

    def fwd(h_over, z_over):
        t = {k: src[k].clone() for k in ("x", "b")}
        h = t[h_over] if h_over else torch.empty_like(t["x"])
        z = t[z_over] if z_over else torch.empty_like(t["x"])
        L.sppo_block_norm_fwd(bn, rows, drop, t["x"], H, t["b"], H, h, H, z, H, cst)
        return [h, z] + [v.clone() for v in st.values()]

    def bwd(dx_over, db_over):
        t = {k: src[k].clone() for k in ("b", "h", "dz", "dh")}
        dx = t[dx_over] if dx_over else torch.empty_like(t["b"])
        db = t[db_over] if db_over else torch.empty_like(t["b"])
        grads = {k: torch.empty_like(v) for k, v in par.items()}
        L.sppo_block_norm_bwd(bn, rows, drop, t["b"], H, t["h"], H, cst, t["dz"], H, t["dh"], H, dx, H, db, H,
                              L.block_norm_grads(**grads), ws, nb, 0)
        return [dx, db] + list(grads.values())

    for v in st.values():
        v.zero_()
    base = fwd(None, None)
    src["h"] = base[0]
    for pair in FWD_ALIASES:
        for i, (u, v) in enumerate(zip(base, fwd(*pair))):
            assert torch.equal(u, v), (pair, i)
    base = bwd(None, None)
    for pair in BWD_ALIASES:
        for i, (u, v) in enumerate(zip(base, bwd(*pair))):
            assert torch.equal(u, v), (pair, i)


def test_block_norm_offset_rows():
    """Rows of mean 1000 and deviation 1 (and one constant row): the squares
    are taken around the mean, so nothing cancels."""
    announce("block norm, large mean")
    c = Case(17, 2048, 2048, "f32", "layer", "layer", "none", True, 0.0, seed=12)
    c.x = c.x * 0.5
    c.b = c.b / 1.5 + 1000.0
    c.b[3] = 1000.0
    h, z = c.forward()
    fwd_check(c, h, z)


def near_back_error(v, e_v, g, e_g, kind, mean, rstd):
    """back_error for a normalised value (v - mean) rstd whose roundings are
    relative to |v - mean|, however far the mean lies."""
    vh = np.abs(v - mean[:, None]) * rstd[:, None]
    m1 = rowmean(np.abs(g)) if kind == "layer" else 0.0
    e1 = rowmean(e_g) + 44 * U * m1 if kind == "layer" else 0.0
    m2 = rowmean(np.abs(g) * vh)
    e2 = rowmean(e_g * vh) + 48 * U * m2
    return rstd[:, None] * (e_g + e1 + vh * e2 + 8 * U * (np.abs(g) + m1 + vh * m2)), vh


@pytest.mark.parametrize("rows,H,dtype,gate,mean", [
    (17, 64, "f32", "channel", 10000.0), (40, 200, "f32", "token", 10000.0), (33, 512, "f32", "none", 10000.0),
    (50, 1024, "f32", "channel", 10000.0), (17, 2048, "f32", "token", 1000.0), (9, 2560, "f32", "channel", 10000.0),
    (20, 8192, "f32", "channel", 10000.0), (40, 1536, "bf16", "channel", 64.0), (12, 5120, "bf16", "token", 64.0),
])
def test_block_norm_backward_of_offset_rows(rows, H, dtype, gate, mean, monkeypatch):
    """Rows whose mean is far larger than their deviation: with the statistics
    as inputs, v - mean loses nothing, so the bounds know no mean."""
    announce(f"block norm backward, large mean rows={rows} H={H} {dtype} {gate} mean={mean}")
    c = Case(rows, H, H, dtype, "layer", "layer", gate, True, 0.1, seed=13)
    c.x = (c.x.float() * 0.5 + mean).to(DT[dtype])
    c.b = (c.b.float() / 1.5 + mean).to(DT[dtype])
    h, _ = c.forward()
    dz, dh = randn(rows, H, H, dtype, 67).cuda(), randn(rows, H, H, dtype, 68).cuda()
    dx, db, g = run_bwd(c, h, dz, dh)
    monkeypatch.setattr(sys.modules[__name__], "back_error", near_back_error)
    bwd_check(c, h, dz, dh, dx, db, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H", [64, 256, 512, 1024, 2048, 4096, 8192])
def test_block_norm_of_constant_rows_is_beta(H, dtype):
    """Rows of one whole number, whose mean is exact at these widths: nothing is
    left of v - mean, and the norm gives its beta, rounded once."""
    announce(f"block norm of constant rows H={H} {dtype}")
    rows = 5
    v = torch.tensor([1000.0, 0.0, -3.0, 129024.0, 1.0])[:, None].expand(rows, H).to(DT[dtype]).contiguous().cuda()
    zero = torch.zeros_like(v)
    gamma, beta = torch.full((H,), 1.5, device="cuda"), torch.linspace(-1, 1, H, device="cuda")
    out, other = torch.empty_like(v), torch.empty_like(v)
    s = [torch.empty(rows, device="cuda") for _ in range(2)]
    L.sppo_block_norm_fwd(L.block_norm(H, dtype, post="layer", post_gamma=gamma, post_beta=beta), rows, None, zero, H,
                          v, H, out, H, None, 0, L.block_norm_stats(post_mean=s[0], post_rstd=s[1]))
    assert torch.equal(out, beta.to(DT[dtype]).expand(rows, H))
    L.sppo_block_norm_fwd(L.block_norm(H, dtype, pre="layer", pre_gamma=gamma, pre_beta=beta), rows, None, v, H,
                          zero, H, other, H, out, H, L.block_norm_stats(pre_mean=s[0], pre_rstd=s[1]))
    assert torch.equal(other, v) and torch.equal(out, beta.to(DT[dtype]).expand(rows, H))


def test_block_norm_gates_only_what_is_kept():
    """No norm after the branch: NaN in dropped places of the branch reaches
    neither h nor the gate's gradient."""
    announce("block norm, NaN in dropped places")
    for gate in ("channel", "token"):
        c = Case(12, 512, 512, "bf16", "none", "layer", gate, True, 0.5, seed=15)
        clean = c.b.clone()
        clean[torch.from_numpy(c.keep == 0)] = 0.0
        c.b = clean
        h, z = c.forward()
        dz, dh = randn(12, 512, 512, "bf16", 63).cuda(), randn(12, 512, 512, "bf16", 64).cuda()
        base = run_bwd(c, h, dz, dh)
        c.b = clean.clone()
        c.b[torch.from_numpy(c.keep == 0)] = float("nan")
        h2, z2 = c.forward()
        assert torch.equal(h, h2) and torch.equal(z, z2)
        got = run_bwd(c, h, dz, dh)
        assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])
        assert torch.equal(got[2]["gate"], base[2]["gate"])


def test_block_norm_drops_what_an_infinite_gate_makes():
    announce("block norm, infinite gate of a row")
    c = Case(8, 256, 256, "bf16", "layer", "none", "token", True, 0.5, seed=16)
    c.dpar["gate"][3] = float("inf")
    h, _ = c.forward()
    want = to_np(c.x)[3, :256]
    dropped = c.keep[3] == 0
    assert np.array_equal(to_np(h)[3][dropped], want[dropped])
    assert not np.isfinite(to_np(h)[3][~dropped]).any()


@pytest.mark.parametrize("rows,H,dtype,post,beta", [
    (5, 64, "f32", "none", False), (7, 256, "bf16", "layer", True), (9, 512, "bf16", "none", False),
    (6, 1024, "f32", "rms", False), (4, 2048, "bf16", "layer", False), (8, 4096, "bf16", "rms", True),
    (3, 8192, "f32", "layer", True), (3, 8192, "bf16", "none", False),
])
def test_block_norm_with_infinite_channel_gates(rows, H, dtype, post, beta):
    """gate n is an infinity of n's sign where a channel's gate is one (NaN
    where n is zero), a dropped element is alpha x, other channels keep their
    bits.  n is known to 1e-5 of its terms, far below the 1e-2 asked for; alpha x
    rounds once before the output does."""
    announce(f"block norm, infinite channel gates rows={rows} H={H} {dtype} {post} beta={beta}")
    c = Case(rows, H, H, dtype, post, "none", "channel", beta, 0.3, 0.75, 0.5, seed=17)
    cols = [0, 5, 9, H - 1]
    c.b[0, 5] = 0.0
    h, _ = c.forward()
    bad = torch.tensor([np.inf, -np.inf, -np.inf, np.inf])
    c.par["gate"][cols] = bad
    c.dpar["gate"][cols] = bad.cuda()
    c.npar["gate"] = to_np(c.par["gate"])
    h2, _ = c.forward()
    rest = torch.ones(H, dtype=torch.bool)
    rest[cols] = False
    assert torch.equal(h[:, rest.cuda()], h2[:, rest.cuda()])
    n = to_np(c.b)
    if post != "none":
        st = c.np_stats()
        n = O._hat(n, st["post_mean"], st["post_rstd"]) * c.npar["post_gamma"] + c.npar.get("post_beta", 0.0)
    with np.errstate(invalid="ignore"):
        ref = 0.75 * to_np(c.x) + 0.5 * O.drop(c.npar["gate"] * n, c.keep)
    ref, n, keep = ref[:, cols], n[:, cols], c.keep[:, cols]
    sure = (keep == 0) | (np.abs(n) > 1e-2) | ((n == 0) & (post == "none"))
    assert sure.mean() > 0.5 and np.isinf(ref[sure]).any()
    within(h2[:, cols][torch.from_numpy(sure).cuda()], ref[sure],
           (HALF[dtype] + 2 * U) * np.abs(np.nan_to_num(ref[sure], posinf=0, neginf=0)), "h")


def test_block_norm_gradient_matches_differences():
    """The fp32 backward along random directions of every input against
    central differences of the kernel's own forward, e = 2^-6: the forward's
    outputs are known to fwd_check's bounds, taken here as 100 u of their
    magnitude, so a difference is off by 2 * 100 u sum(|w| |out|) / (2 e) at
    worst, and by the truncation that the oracle's own difference shows."""
    announce("block norm against differences")
    rows, H = 6, 64
    c = Case(rows, H, H, "f32", "layer", "rms", "channel", True, 0.25, 0.8, 0.7, seed=20)
    dz, dh = randn(rows, H, H, "f32", 70), randn(rows, H, H, "f32", 71)
    h, z = c.forward()
    dx, db, g = run_bwd(c, h, dz.cuda(), dh.cuda())
    grads = {"x": to_np(dx), "b": to_np(db), **{k: to_np(v) for k, v in g.items()}}
    e = 2.0 ** -6
    wz, wh = to_np(dz), to_np(dh)

    def outputs(name, sign, d):
        k = Case(rows, H, H, "f32", "layer", "rms", "channel", True, 0.25, 0.8, 0.7, seed=20)
        if name in ("x", "b"):
            setattr(k, name, getattr(k, name) + sign * e * d)
            args = to_np(k.x), to_np(k.b), k.npar
        else:
            k.par[name] = k.par[name] + sign * e * d
            k.dpar[name] = k.par[name].cuda()
            k.npar[name] = to_np(k.par[name])
            k.bn = L.block_norm(H, "f32", "layer", "rms", "channel", 1e-5, 0.8, 0.7, **k.dpar)
            args = to_np(k.x), to_np(k.b), k.npar
        hh, zz = k.forward()
        r = O.block_norm_fwd(args[0], args[1], k.cfg, args[2], k.keep)
        return to_np(hh), to_np(zz), (wz * r["z"]).sum() + (wh * r["h"]).sum()

    for name in grads:
        shape = grads[name].shape
        d = torch.randn(shape, generator=torch.Generator().manual_seed(5))
        hu, zu, ou = outputs(name, 1, d)
        hd, zd, od = outputs(name, -1, d)
        diff = ((wz * (zu - zd)).sum() + (wh * (hu - hd)).sum()) / (2 * e)
        along = (grads[name] * to_np(d)).sum()
        f = O.block_norm_fwd(to_np(c.x), to_np(c.b), c.cfg, c.npar, c.keep)
        og = O.block_norm_bwd(to_np(c.b), f["h"], f, wz, wh, c.cfg, c.npar, c.keep)
        exact = (og[{"x": "dx", "b": "db"}.get(name, name)] * to_np(d)).sum()
        trunc = abs((ou - od) / (2 * e) - exact)
        noise = 100 * U * (np.abs(wz * zu).sum() + np.abs(wh * hu).sum()) / e
        assert abs(diff - along) <= trunc + noise + 1e-4 * np.abs(grads[name] * to_np(d)).sum(), (name, diff, along)


def test_block_norm_graphs_and_streams():
    """Forward and backward captured twice, each graph with its own buffers,
    replayed at once on two streams and between eager calls: every replay has
    the eager bits."""
    announce("block norm in two graphs")
    sides = []
    for i in range(2):
        c = Case(300 + i, 1536, 1536, "bf16", "layer", "layer", "channel", True, 0.1, seed=30 + i)
        c.x, c.b = c.x.cuda(), c.b.cuda()
        H, rows = c.H, c.rows
        h, z = c.act(), c.act()
        dz, dh = randn(rows, H, H, "bf16", 80 + i).cuda(), randn(rows, H, H, "bf16", 81 + i).cuda()
        dx, db = c.act(), c.act()
        g = {k: torch.empty_like(v) for k, v in c.dpar.items()}
        nb = L.sppo_block_norm_bwd_workspace(c.bn, rows)
        ws = torch.empty(nb // 4, device="cuda")
        gr = L.block_norm_grads(**g)

        def work(c=c, H=H, rows=rows, h=h, z=z, dz=dz, dh=dh, dx=dx, db=db, nb=nb, ws=ws, gr=gr):
            L.sppo_block_norm_fwd(c.bn, rows, c.drop, c.x, H, c.b, H, h, H, z, H, c.cstats)
            L.sppo_block_norm_bwd(c.bn, rows, c.drop, c.b, H, h, H, c.cstats, dz, H, dh, H, dx, H, db, H, gr, ws, nb, 0)

        outs = [h, z, dx, db] + list(g.values())
        work()
        torch.cuda.synchronize()
        ref = [t.clone() for t in outs]
        s = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work()
        sides.append((graph, s, outs, ref, work, (c, ws, gr, g)))
    for _ in range(4):
        for _, _, outs, _, _, _ in sides:
            for t in outs:
                t.zero_()
        torch.cuda.synchronize()
        for graph, s, *_ in sides:
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for _, _, outs, ref, _, _ in sides:
            for a, b in zip(outs, ref):
                assert torch.equal(a, b)
        sides[0][4]()  # an eager run between the replays
        torch.cuda.synchronize()


# ------------------------------------------------------------------ embedding
def make_ids(rows, V, kind, seed):
    g = np.random.default_rng(seed)
    if kind == "same":
        ids = np.full(rows, V // 2)
    elif kind == "distinct":
        ids = g.permutation(V)[:rows] if rows <= V else g.permutation(rows) % V
    elif kind == "zipf":
        ids = np.minimum(np.exp(g.random(rows) * np.log(V + 1.0)).astype(np.int64) - 1, V - 1)
    elif kind == "runs":  # every run length from 1 to 40 and longer ones, rows shuffled
        n = g.integers(1, 41, size=rows)
        n[::9] *= 5
        ids = g.permutation(np.repeat(np.arange(rows), n)[:rows] % V)
    else:  # padding and ids of other ranks' parts, also past 32 bits
        ids = g.integers(-3, V + 3, size=rows)
    return ids.astype(np.int64)


EMBED_CASES = [
    # rows, H, V, dtype, id type, ids, p, scale
    (1, 8, 1, "bf16", "i64", "same", 0.0, 1.0),
    (1, 64, 1000, "f32", "i32", "zipf", 0.5, 3.0),
    (33, 264, 7, "bf16", "i32", "outside", 0.1, 64.0),
    (257, 2056, 500, "bf16", "i64", "zipf", 0.1, 8.0),
    (31, 8192, 40, "f32", "i64", "distinct", 0.0, 1.0),
    (64, 128, 64, "bf16", "i64", "same", 0.2, 1.0),
    (3000, 72, 300, "bf16", "i64", "same", 0.0, 2.0),      # one run over every tile
    (5000, 40, 50000, "f32", "i64", "distinct", 0.0, 1.0),
    (4099, 256, 33000, "bf16", "i32", "zipf", 0.1, 1.0),
    (300001, 8, 300000, "bf16", "i64", "zipf", 0.0, 1.0),  # three passes of the sort, several steps a tile
    (150000, 16, 3, "f32", "i32", "outside", 0.3, 1.0),
    (4096, 24, 4096, "bf16", "i32", "runs", 0.0, 1.0),     # the ranking with 4, 2 and 1 lanes a row
    (8191, 16, 9000, "f32", "i64", "runs", 0.0, 1.0),
    (16384, 8, 20000, "f32", "i64", "runs", 0.0, 1.0),
    (6000, 520, 9, "bf16", "i64", "outside", 0.1, 1.0),    # runs over many groups
    (3000, 1032, 60, "f32", "i64", "zipf", 0.0, 1.0),
    (16385, 512, 20000, "bf16", "i64", "runs", 0.0, 1.0),  # one more than it takes
    (17, 16, 4, "f32", "i64", "same", 0.0, 1.0),
    (256, 520, 4, "bf16", "i32", "same", 0.1, 1.0),        # the most rows without a sorted list, one run
    (255, 24, 90, "f32", "i64", "runs", 0.0, 1.0),
    (200, 1032, 300, "bf16", "i64", "outside", 0.1, 1.0),
    (257, 16, 4, "f32", "i64", "same", 0.0, 1.0),          # one more
    (1024, 520, 70, "bf16", "i64", "runs", 0.1, 1.0),
    (1000, 16, 300, "f32", "i32", "outside", 0.0, 1.0),
    (1025, 16, 4, "f32", "i64", "same", 0.0, 1.0),
    (4100, 4096, 900, "bf16", "i64", "zipf", 0.1, 1.0),    # read past the caches
    (33000, 256, 5000, "f32", "i64", "runs", 0.0, 1.0),
]


@pytest.mark.parametrize("rows,H,V,dtype,idt,kind,p,scale", EMBED_CASES)
def test_embedding(rows, H, V, dtype, idt, kind, p, scale):
    announce(f"embedding rows={rows} H={H} V={V} {dtype} {idt} {kind} p={p}")
    ids = make_ids(rows, V, kind, rows + H)
    if kind == "outside" and idt == "i64":
        ids[::5] += 2 ** 32
    dids = torch.from_numpy(ids).to(torch.int32 if idt == "i32" else torch.int64).cuda()
    ld, ldt = H + 8, H + 16
    table = randn(V, H, ldt, dtype, 1)
    seed, row0 = 99, 10 ** 6
    drop = L.drop_spec(p, seed, 4, row0) if p > 0 else None
    keep = O.keep_factor(rows, H, p, seed, 4, row0) if p > 0 else np.ones((rows, H))
    y = torch.full((rows, ld), 7.0, device="cuda", dtype=DT[dtype])
    L.sppo_embedding_fwd(rows, H, V, dids, table.cuda(), ldt, scale, drop, y, ld, dtype, idt)
    ref = O.embedding_fwd(ids, to_np(table)[:, :H], scale, keep)
    within(y[:, :H], ref, (HALF[dtype] + 4 * U) * np.abs(ref), "y")  # scale, keep factor, two products
    assert torch.all(y[:, H:] == 7.0)
    # gradient: written over everything, then added
    dy = randn(rows, H, ld, dtype, 2)
    dyd = dy.cuda()
    dt = torch.full((V, ldt), 7.0, device="cuda")
    nb = L.sppo_embedding_bwd_workspace(rows, H)
    ws = torch.full((nb,), 0xA5, dtype=torch.uint8, device="cuda")
    call = lambda t, acc: L.sppo_embedding_bwd(rows, H, V, dids, dyd, ld, scale, drop, t, ldt, ws, nb, acc, dtype, idt)
    call(dt, 0)
    g = to_np(dy)[:, :H]
    ref = O.embedding_bwd(ids, g, V, scale, keep)
    # a wave's 31 rows at most one by one, four waves, groups of 64 rows in four
    # rows of them and those, and 8 roundings more
    tol = (31 + 4 + -(-rows // 256) + 4 + 8) * U * O.embedding_bwd(ids, np.abs(g), V, abs(scale), keep)
    within(dt[:, :H], ref, tol, "dtable")
    assert torch.all(dt[:, H:] == 7.0)
    again = torch.full((V, ldt), 7.0, device="cuda")
    call(again, 0)
    assert torch.equal(dt, again), "the same bits again"
    base = torch.randn(V, ldt, generator=torch.Generator().manual_seed(3))
    acc = base.cuda()
    call(acc, 1)
    within(acc[:, :H], to_np(base)[:, :H] + ref, tol + U * np.abs(to_np(base)[:, :H] + ref), "accumulated")
    absent = torch.from_numpy(np.setdiff1d(np.arange(V), ids))
    assert torch.equal(acc[absent.cuda()].cpu(), base[absent]), "rows without a token changed"
    assert torch.equal(acc[:, H:].cpu(), base[:, H:])


def test_embedding_gradient_of_one_token_in_all_rows():
    """2^21 rows of one token, columns of one value each: equal partial sums of
    one sign, whose roundings in a plain chain add up (400 to 1400 u here).  16
    rows, 4 waves, then 64, 64 and 2 sums in turn, 4 chains and the scale."""
    rows, H, V = 2 ** 21, 8, 3
    announce(f"embedding gradient, rows={rows} of one token")
    vals = torch.tensor([1.2345678, 1.7, 1.1, 1.9999, 1.3, 1.45, -1.7, -1.3])
    dy = vals.expand(rows, H).contiguous().cuda()
    ids = torch.ones(rows, dtype=torch.int32, device="cuda")
    ws = torch.empty(L.sppo_embedding_bwd_workspace(rows, H), dtype=torch.uint8, device="cuda")
    dt = torch.full((V, H), 7.0, device="cuda")
    L.sppo_embedding_bwd(rows, H, V, ids, dy, H, 1.0, None, dt, H, ws, ws.numel(), 0, "f32", "i32")
    ref = to_np(vals) * rows
    within(dt[1], ref, (16 + 4 + 64 + 64 + 2 + 4 + 1) * U * np.abs(ref), "dtable")
    assert torch.all(dt[::2] == 0)


def test_embedding_rows_outside_read_nothing():
    """NaN in the rows of dy whose ids lie outside reaches no gradient, and a
    table of NaN no output row of such an id."""
    announce("embedding, padding")
    rows, H, V = 100, 64, 10
    ids = torch.from_numpy(make_ids(rows, V, "outside", 5)).cuda()
    out = (ids < 0) | (ids >= V)
    dy = randn(rows, H, H, "bf16", 8).cuda()
    clean = dy.clone()
    clean[out] = 0.0
    dy[out] = float("nan")
    nb = L.sppo_embedding_bwd_workspace(rows, H)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    a, b = torch.empty(V, H, device="cuda"), torch.empty(V, H, device="cuda")
    L.sppo_embedding_bwd(rows, H, V, ids, dy, H, 1.0, None, a, H, ws, nb, 0)
    L.sppo_embedding_bwd(rows, H, V, ids, clean, H, 1.0, None, b, H, ws, nb, 0)
    assert torch.equal(a, b) and torch.isfinite(a).all()
    y = torch.empty(rows, H, device="cuda", dtype=BF)
    L.sppo_embedding_fwd(rows, H, V, ids, torch.full((V, H), float("nan"), device="cuda", dtype=BF), H, 1.0,
                         L.drop_spec(0.1, 1), y, H)
    assert torch.all(y[out] == 0)


def test_embedding_past_a_launch():
    """A lookup of more elements than one launch takes (2^33): rows at both
    ends and around the boundary."""
    announce("embedding of 2^33 elements")
    H, V = 16384, 64
    rows = 2 ** 33 // H + 3
    ids = torch.arange(rows, device="cuda") % (V + 1)
    table = randn(V, H, H, "bf16", 9).cuda()
    y = torch.full((rows, H), 7.0, device="cuda", dtype=BF)
    L.sppo_embedding_fwd(rows, H, V, ids, table, H, 2.0, L.drop_spec(0.25, 13, 1, 5), y, H)
    for r in (0, 1, V, rows // 2, rows - 4, rows - 3, rows - 2, rows - 1):
        ref = O.embedding_fwd(np.array([r % (V + 1)]), to_np(table), 2.0, O.keep_factor(1, H, 0.25, 13, 1, row0=5 + r))
        within(y[r:r + 1], ref, (HALF["bf16"] + 4 * U) * np.abs(ref), r)


@pytest.mark.parametrize("rows", [100, 700, 9000])  # each way to order the rows
def test_embedding_gradient_in_graphs(rows):
    """Two captured gradients with a workspace each, replayed at once on two
    streams with new tokens in between: every replay has the eager bits."""
    announce(f"embedding gradient in two graphs, rows={rows}")
    H, V = 512, 90
    sides = []
    for i in range(2):
        ids = torch.from_numpy(make_ids(rows, V, "zipf", i)).cuda()
        dy = randn(rows, H, H, "bf16", 90 + i).cuda()
        dt = torch.zeros(V, H, device="cuda")
        nb = L.sppo_embedding_bwd_workspace(rows, H)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")

        def work(ids=ids, dy=dy, dt=dt, nb=nb, ws=ws, acc=i):
            L.sppo_embedding_bwd(rows, H, V, ids, dy, H, 1.5, None, dt, H, ws, nb, acc)

        s = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work()
        sides.append((graph, s, ids, dt, work, ws, dy))
    for n in range(4):
        for i, (_, _, ids, dt, *_) in enumerate(sides):
            ids.copy_(torch.from_numpy(make_ids(rows, V, "zipf", 10 * n + i)))
            dt.fill_(0.25)
        torch.cuda.synchronize()
        for graph, s, *_ in sides:
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        got = [t[3].clone() for t in sides]
        for t, x in zip(sides, got):
            t[3].fill_(0.25)
            t[4]()
            torch.cuda.synchronize()
            assert torch.equal(t[3], x)


def test_calls_without_a_stream_run_on_the_current_one():
    """A call without a stream inside torch.cuda.stream(s) goes to s: it waits
    for what s holds (a long copy), not for the default stream."""
    announce("current stream")
    from paper_2503_10377_amd.sppo import _stream
    s = torch.cuda.Stream()
    assert _stream(None) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(s):
        assert _stream(None) == s.cuda_stream
        x = torch.ones(1 << 26, device="cuda", dtype=BF)
        y = x * 2
        z = torch.empty_like(x)
        L.sppo_dropout(1 << 12, 1 << 14, y, 1 << 14, L.drop_spec(0.0, 0), z, 1 << 14)
    s.synchronize()
    assert torch.all(z == 2)
