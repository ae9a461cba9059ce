"""The operators that close a training step on the GPU against the fp64 oracle:
rotary positions, cross-entropy with its gradient, the gradient norm, AdamW
with states in 32 and in 8 bits.

Tolerances count roundings.  u = 2^-24 is half a step of fp32, half(t) that of
the output's type (bf16 2^-8, fp32 2^-24), relative to the value.
"""
import sys

import numpy as np
import pytest
import torch

from oracle import step_ops as O
from paper_2503_10377_amd import sppo as L
from parity import to_np

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF, "f32": F32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
IDS = {"i32": torch.int32, "i64": torch.int64}
U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")


def announce(msg):
    print(f"\n[case] {msg}", file=sys.stderr, flush=True)


def randn(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale


def within(got, ref, tol, what):
    """|got - ref| <= tol, element by element (NaN and infinities alike)."""
    got, ref = to_np(got), np.asarray(ref)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - ref) <= tol))
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(),
                           got[bad][:3], ref[bad][:3], np.broadcast_to(tol, ref.shape)[bad][:3])


# ------------------------------------------------------------------- rotary
def table(rot, **kw):
    freqs, amp = L.sppo_rotary_freqs(rot, **kw)
    return freqs, torch.from_numpy(np.array(freqs, dtype=np.uint64).view(np.int64)).cuda(), amp


def rotary_check(y, x, pos, freqs, rot, layout, amp, inverse, dtype, what):
    """The angle rounds twice (u pi/4 each), a cosine or sine three times more
    (series, amplitude), the two products and their sum once each: below 8 u of
    amp (|a| + |b|), of which a pair's members have at most sqrt(2) of its
    length."""
    x = to_np(x)
    ref = O.rotary(x, pos, freqs, rot, layout, amp, inverse)
    flat = np.ones_like(x)
    i = np.arange(rot // 2)
    ia, ib = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    flat[...] = 0.0
    flat[..., ia] = flat[..., ib] = np.abs(x[..., ia]) + np.abs(x[..., ib])
    tol = HALF[dtype] * np.abs(ref) + 8 * U * abs(amp) * flat
    tol[..., rot:] = 0.0
    within(y, ref, tol, what)


@pytest.mark.parametrize("rows,hq,hk,D,rot,layout,dtype,kdtype,pos,row0,inv,kw,pad", [
    (1, 32, 8, 128, 128, "half", "bf16", "bf16", "i64", 0, 0, {}, 0),
    (1, 1, 1, 8, 8, "half", "f32", "f32", None, 0, 0, {}, 0),
    (3, 2, 1, 64, 24, "half", "bf16", "f32", None, 2 ** 31, 1, {}, 8),       # pieces of four, copied ends
    (37, 5, 3, 96, 96, "interleaved", "f32", "bf16", "i32", 0, 0, dict(scaling="ntk", factor=8.0), 24),
    (130, 32, 32, 128, 64, "interleaved", "bf16", "bf16", None, 10 ** 6 + 3, 1,
     dict(scaling="yarn", factor=8.0, original_len=4096), 0),
    (257, 7, 1, 256, 256, "half", "bf16", "f32", "i64", 0, 0, dict(scaling="linear", factor=3.0), 128),
    (9, 3, 2, 1024, 1024, "interleaved", "f32", "f32", None, -5, 0, {}, 0),  # positions below zero
    (5, 2, 2, 72, 16, "half", "bf16", "bf16", None, 2 ** 62, 1, dict(base=500000.0), 0),
])
def test_rotary(rows, hq, hk, D, rot, layout, dtype, kdtype, pos, row0, inv, kw, pad):
    announce(f"rotary rows={rows} heads={hq},{hk} D={D} rot={rot} {layout} {dtype},{kdtype} pos={pos} row0={row0} "
             f"inverse={inv} {kw} pad={pad}")
    freqs, dev, amp = table(rot, **kw)
    at = np.arange(rows).astype(object) + row0
    p = None
    if pos is not None:
        p = torch.randint(-1000, 2 ** 31 - 1, (rows,), generator=torch.Generator().manual_seed(3)).to(IDS[pos])
        if pos == "i64":
            p = p * 2 ** 20 + 7
        at = p.tolist()
        p = p.cuda()
    spec = L.rotary(rot, dev, layout, amp, row0, p, pos or "i64")
    xs, ys, ts = [], [], []
    for n, (h, dt) in enumerate(((hq, dtype), (hk, kdtype))):
        x = randn((rows, h * D + pad), 10 + n).to(DT[dt]).cuda()
        y = torch.full((rows, h * D + pad + 8), 7.0, device="cuda", dtype=DT[dt])
        ts.append(L.rotary_tensor(h, D, x, h * D + pad, D, y, h * D + pad + 8, D, dt))
        xs.append(x)
        ys.append(y)
    L.sppo_rotary_apply(spec, rows, L.rotary_tensors(ts), inv)
    for x, y, h, dt in zip(xs, ys, (hq, hk), (dtype, kdtype)):
        rotary_check(y[:, :h * D].reshape(rows, h, D), x[:, :h * D].reshape(rows, h, D), at, freqs, rot, layout, amp,
                     inv, dt, "y")
        assert torch.all(y[:, h * D:] == 7.0), "columns past the heads written"


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_in_place_head_major_and_in_chunks(layout):
    """The same bits in place, from a head-major tensor, in chunks of the
    sequence, with the positions given, and for four tensors at once."""
    rows, h, D, rot = 77, 5, 64, 48
    announce(f"rotary in place, head-major, chunks {layout}")
    _, dev, amp = table(rot)
    x = randn((rows, h, D), 1).to(BF).cuda()
    spec = lambda row0, p=None: L.rotary(rot, dev, layout, amp, row0, p)  # noqa: E731
    one = lambda a, b, n=h * D, hs=D: L.rotary_tensor(h, D, a, n, hs, b, n, hs)  # noqa: E731
    whole = torch.empty_like(x)
    L.sppo_rotary_apply(spec(1000), rows, L.rotary_tensors([one(x, whole)]))
    y = x.clone()
    L.sppo_rotary_apply(spec(1000), rows, L.rotary_tensors([one(y, y)]))
    assert torch.equal(y, whole)
    xt = x.transpose(0, 1).contiguous()
    yt = torch.empty_like(xt)
    L.sppo_rotary_apply(spec(1000), rows, L.rotary_tensors([one(xt, yt, D, rows * D)]))
    assert torch.equal(yt.transpose(0, 1), whole)
    parts = [torch.empty_like(x) for _ in range(4)]
    for c0, c1 in ((0, 1), (1, 40), (40, 77)):
        L.sppo_rotary_apply(spec(1000 + c0), c1 - c0, L.rotary_tensors([one(x[c0:], q[c0:]) for q in parts]))
    p = torch.arange(1000, 1000 + rows, device="cuda")
    given = torch.empty_like(x)
    L.sppo_rotary_apply(spec(0, p), rows, L.rotary_tensors([one(x, given)]))
    for q in parts + [given]:
        assert torch.equal(q, whole)


def test_rotary_inverse_is_the_gradient():
    """<R x, w> = <x, R' w> on fp32, and central differences of it (the rotation is
    linear: they are exact but for rounding)."""
    rows, h, D = 6, 2, 32
    announce("rotary gradient")
    _, dev, amp = table(16, scaling="yarn", factor=4.0, original_len=64)
    x, w = randn((rows, h, D), 1).cuda(), randn((rows, h, D), 2).cuda()
    spec = L.rotary(16, dev, "interleaved", amp, 12345)

    def turn(v, inverse):
        y = torch.empty_like(v)
        L.sppo_rotary_apply(spec, rows, L.rotary_tensors([L.rotary_tensor(h, D, v, h * D, D, y, h * D, D, "f32")]),
                            inverse)
        return y

    g = to_np(turn(w, 1)).ravel()
    f = lambda v: float((to_np(turn(v, 0)) * to_np(w)).sum())  # noqa: E731
    for i in range(0, x.numel(), 29):
        d = torch.zeros_like(x).view(-1)
        d[i] = 1.0
        d = d.view_as(x)
        # Differences over two units, of sums whose terms are off by 16 u of |x| + 1, |w| each.
        err = 16 * U * float((np.abs(to_np(x)) + 1).sum() * np.abs(to_np(w)).max()) * 2
        assert abs((f(x + d) - f(x - d)) / 2 - g[i]) <= err


# --------------------------------------------------------------------- loss
def ce_tol(x, t, V, ref, smooth, z, scale, dtype, lse_in=None, dloss=None):
    """(loss, lse, dx) tolerances.  A difference x - max rounds once, its product
    with log2(e) twice (3 u of the row's range R), exp2 to 2 u; the sum is added
    up over at most 64 + 4 V / 8192 additions and rescalings, each change of the
    running maximum with the same errors again: S is off by (6 R + 66 + 4 V /
    8192) u of itself, lse by that and its own roundings."""
    x = np.asarray(x, dtype=np.float64)
    loss, lse, dx = ref
    with np.errstate(all="ignore"):
        fin = np.where(np.isfinite(x), x, np.nan)
        top = np.nanmax(fin, axis=1)
        R = top - np.nanmin(fin, axis=1)
        s = U * (6 * R + 66 + 4 * V / 8192)
        part = np.abs(lse - top)
        tol_lse = s + U * (2 * part + 2 * np.abs(lse))
        xt = x[np.arange(len(x)), np.clip(t, 0, V - 1)]
        mean = np.nanmean(np.abs(fin), axis=1)
        tol_loss = s + U * (4 * (np.abs(top - xt) + part) + smooth * (80 + V / 2048) * (mean + np.abs(top))
                            + 2 * np.abs(loss)) + 2 * z * np.abs(lse) * tol_lse + 8 * U * z * lse ** 2
        if lse_in is not None:
            R, s = np.nanmax(np.abs(fin - lse[:, None]), axis=1), 0.0
        w = np.abs(scale) * (1.0 if dloss is None else np.abs(dloss))
        p = np.abs(1.0 + 2 * z * lse)[:, None] * np.minimum(np.exp(x - lse[:, None]), 1.0)
        rel = U * (3 * R + 12) + s
        hit = np.zeros_like(x)
        ok = (t >= 0) & (t < V)
        hit[np.arange(len(x))[ok], t[ok]] = 1.0
        tol_dx = (w * rel)[:, None] * p + (4 * U * w * np.ones(len(x)))[:, None] * (p + hit + smooth / V) \
            + HALF[dtype] * np.abs(dx) + 2.0 ** -126
    return tol_loss, tol_lse, tol_dx


def ce_inputs(rows, V, ld, dtype, seed, ids="i64", padded=(), dead=0, scale=3.0, shift=0.0):
    x = (randn((rows, ld), seed, scale) + shift).to(DT[dtype])
    if dead:
        x[:, V - dead:V] = -INF
    t = torch.randint(0, V - dead, (rows,), generator=torch.Generator().manual_seed(seed + 1))
    for i, bad in zip(range(0, rows, 3), padded):
        t[i] = bad
    return x, t.to(IDS[ids])


def workspace(ce, rows):
    n = L.sppo_cross_entropy_workspace(ce, rows)
    return torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda"), n


def run_ce(ce, rows, x, ld, t, dtype, in_place=False, grad=True):
    loss, lse = (torch.full((rows,), 9.0, device="cuda") for _ in range(2))
    dx = (x if in_place else torch.full((rows, ld), 7.0, device="cuda", dtype=DT[dtype])) if grad else None
    ws, n = workspace(ce, rows)
    L.sppo_cross_entropy(ce, rows, x, ld, t, loss, lse, dx, ld, ws, n)
    return loss, lse, dx


CE_SIZES = [
    (1, 1, 8, "bf16"), (1, 2, 8, "f32"), (3, 7, 16, "bf16"), (5, 8, 8, "f32"), (70, 63, 64, "bf16"),
    (33, 1000, 1008, "f32"), (4, 2048, 2048, "bf16"), (4, 2049, 2056, "bf16"), (19, 8191, 8192, "f32"),
    (6, 16391, 16400, "bf16"), (7, 32768, 32768, "bf16"), (5, 32777, 32784, "f32"), (3, 65536, 65536, "bf16"),
    (3, 65537, 65544, "f32"), (2, 131072, 131072, "bf16"), (2, 131081, 131088, "bf16"), (1, 300007, 300016, "f32"),
    (1, 262144, 262144, "bf16"), (600, 300, 304, "bf16"), (700, 4099, 4104, "f32"), (300, 70001, 70008, "bf16"),
]


@pytest.mark.parametrize("rows,V,ld,dtype", CE_SIZES)
@pytest.mark.parametrize("smooth,z", [(0.0, 0.0), (0.1, 1e-3)])
def test_cross_entropy(rows, V, ld, dtype, smooth, z):
    announce(f"cross entropy rows={rows} V={V} ld={ld} {dtype} smooth={smooth} z={z}")
    ids = "i32" if V % 2 else "i64"
    x, t = ce_inputs(rows, V, ld, dtype, 5, ids, padded=() if rows == 1 else (-1, V, 2 ** 31 - 1, -2 ** 31),
                     shift=40.0)
    scale_dev = torch.tensor([0.25], device="cuda")
    ce = L.cross_entropy(V, dtype, ids, smooth, z, 0.5, scale_dev)
    loss, lse, dx = run_ce(ce, rows, x.cuda(), ld, t.cuda(), dtype)
    ref = O.cross_entropy(to_np(x)[:, :V], t.numpy(), smooth, z, 0.125)
    tol = ce_tol(to_np(x)[:, :V], t.numpy().astype(np.int64), V, ref, smooth, z, 0.125, dtype)
    within(loss, ref[0], tol[0], "loss")
    within(lse, ref[1], tol[1], "lse")
    within(dx[:, :V], ref[2], tol[2], "dx")
    assert torch.all(dx[:, V:] == 7.0), "columns past V written"
    # The loss alone, the gradient over the logits, and the gradient from the kept lse.
    alone, lse2, _ = run_ce(ce, rows, x.cuda(), ld, t.cuda(), dtype, grad=False)
    assert torch.equal(alone, loss) and torch.equal(lse2, lse)
    over = x.cuda()
    run_ce(ce, rows, over, ld, t.cuda(), dtype, in_place=True)
    assert torch.equal(over[:, :V], dx[:, :V]) and torch.equal(over[:, V:].cpu(), x[:, V:])
    dloss = randn((rows,), 8).cuda()
    ref = O.cross_entropy(to_np(x)[:, :V], t.numpy(), smooth, z, 0.125, to_np(lse), to_np(dloss))
    tol = ce_tol(to_np(x)[:, :V], t.numpy().astype(np.int64), V, ref, smooth, z, 0.125, dtype, to_np(lse), to_np(dloss))
    back = torch.full((rows, ld), 7.0, device="cuda", dtype=DT[dtype])
    L.sppo_cross_entropy_bwd(ce, rows, x.cuda(), ld, t.cuda(), lse, dloss, back, ld)
    within(back[:, :V], ref[2], tol[2], "dx from lse")
    assert torch.all(back[:, V:] == 7.0), "columns past V written"


@pytest.mark.parametrize("V,dtype", [(9, "f32"), (3000, "bf16"), (40007, "bf16"), (200003, "f32")])
def test_cross_entropy_of_masked_logits(V, dtype):
    """Masked classes, a target at one, rows of nothing else, NaN; rows without a
    target whatever they hold."""
    announce(f"cross entropy of masked logits V={V} {dtype}")
    ld = (V + 7) // 8 * 8
    x, t = ce_inputs(8, V, ld, dtype, 3, scale=1.0)
    x[1, 1:V] = -INF           # one class left
    t[1] = 0
    x[2, :V // 2] = -INF
    t[2] = 0                   # the target is masked
    x[3, :V] = -INF            # nothing left
    x[4, V // 2] = NAN
    x[5, :V], t[5] = NAN, -1   # ignored
    x[6, :V], t[6] = -INF, V   # ignored
    x[7, :V] = -1e30           # far below, but not masked
    ce = L.cross_entropy(V, dtype, scale=2.0)
    loss, lse, dx = run_ce(ce, 8, x.cuda(), ld, t.cuda(), dtype)
    ref = O.cross_entropy(to_np(x)[:, :V], t.numpy(), scale=2.0)
    assert lse[3] == -INF and loss[2] == INF and ref[0][2] == INF
    assert torch.isnan(loss[3:5]).all() and torch.isnan(lse[4]) and torch.isnan(dx[3:5, :V]).all()
    for r in (5, 6):
        assert loss[r] == 0 and lse[r] == 0 and not dx[r, :V].any()
    assert loss[1] == 0 and torch.all(dx[1, :V] == 0)
    keep = [0, 1, 2, 7]
    sub = [a[keep] for a in ref]
    tol = ce_tol(to_np(x)[keep][:, :V], t.numpy()[keep], V, sub, 0.0, 0.0, 2.0, dtype)
    within(loss[keep], sub[0], tol[0], "loss")
    within(lse[keep], sub[1], tol[1], "lse")
    within(dx[keep][:, :V], sub[2], tol[2], "dx")
    back = torch.empty_like(dx)
    L.sppo_cross_entropy_bwd(ce, 8, x.cuda(), ld, t.cuda(), lse, None, back, ld)
    assert torch.isnan(back[3:5, :V]).all() and not back[5:7, :V].any()
    # With smoothing a masked class makes the loss infinite, a masked target too.
    loss, _, _ = run_ce(L.cross_entropy(V, dtype, label_smoothing=0.5), 8, x.cuda(), ld, t.cuda(), dtype)
    assert loss[1] == INF and loss[2] == INF and loss[5] == 0 and torch.isfinite(loss[0])


@pytest.mark.parametrize("V,dtype", [(100, "bf16"), (50000, "f32"), (140000, "bf16")])
def test_cross_entropy_of_infinite_logits(V, dtype):
    """A logit of +inf: lse and the loss of any other target are +inf, its own
    gradient is NaN, the others' is the formula's at probability zero."""
    announce(f"cross entropy of +inf V={V} {dtype}")
    ld = (V + 7) // 8 * 8
    x, t = ce_inputs(2, V, ld, dtype, 3, scale=100.0)
    x[:, V // 3] = INF
    t[0], t[1] = 5, V // 3
    loss, lse, dx = run_ce(L.cross_entropy(V, dtype, scale=2.0), 2, x.cuda(), ld, t.cuda(), dtype)
    assert torch.all(lse == INF) and loss[0] == INF and torch.isnan(loss[1])
    want = torch.zeros(2, V)
    want[0, 5] = -2.0
    want[:, V // 3] = NAN
    within(dx[:, :V], to_np(want), 0.0, "dx")


def test_calls_past_32_bit_offsets():
    """Rows and elements whose offsets pass 2^32, in a buffer that is touched at
    few places."""
    announce("offsets past 2^32")
    rows, ld = 4100, 1 << 20
    buf = torch.empty(rows * ld, dtype=BF, device="cuda").view(rows, ld)
    freqs, dev, amp = table(64)
    x = randn((rows, 64), 1).to(BF)
    buf[:, :64] = x.cuda()
    L.sppo_rotary_apply(L.rotary(64, dev, "half", amp), rows,
                        L.rotary_tensors([L.rotary_tensor(1, 64, buf, ld, 64, buf, ld, 64)]))
    rotary_check(buf[:, :64].reshape(rows, 1, 64), x.reshape(rows, 1, 64), range(rows), freqs, 64, "half", amp, 0,
                 "bf16", "y")
    for V in (100, 40001):
        n = rows if V == 100 else 4100
        x, t = ce_inputs(n, V, V + 7 & ~7, "bf16", 2)
        buf[:n, :x.shape[1]] = x.cuda()
        pick = [0, 1, n - 2, n - 1]
        loss, lse, _ = run_ce(L.cross_entropy(V), n, buf, ld, t.cuda(), "bf16", in_place=True)
        sub, tt = to_np(x)[pick][:, :V], t.numpy()[pick]
        ref = O.cross_entropy(sub, tt)
        tol = ce_tol(sub, tt, V, ref, 0.0, 0.0, 1.0, "bf16")
        within(loss[pick], ref[0], tol[0], "loss")
        within(buf[pick][:, :V], ref[2], tol[2], "dx")
        buf[:n, :x.shape[1]] = x.cuda()
        L.sppo_cross_entropy_bwd(L.cross_entropy(V), n, buf, ld, t.cuda(), lse, None, buf, ld)
        within(buf[pick][:, :V], ref[2], tol[2] + 8 * U * np.abs(ref[1])[:, None], "dx from lse")


def test_calls_past_a_launch():
    """More rows than one launch takes (2^25 waves): rows at both sides of the
    border and at the end."""
    rows = (1 << 25) + 5
    announce("calls past a launch")
    pick = torch.tensor([0, 1, 2 ** 25 - 1, 2 ** 25, 2 ** 25 + 1, rows - 1])
    x = torch.randn(rows, 8, device="cuda").to(BF)
    freqs, dev, amp = table(8)
    y = torch.empty_like(x)
    L.sppo_rotary_apply(L.rotary(8, dev, "half", amp, 3), rows,
                        L.rotary_tensors([L.rotary_tensor(1, 8, x, 8, 8, y, 8, 8)]))
    rotary_check(y[pick].reshape(-1, 1, 8), x[pick].reshape(-1, 1, 8), (pick + 3).tolist(), freqs, 8, "half", amp, 0,
                 "bf16", "y")
    t = torch.randint(0, 7, (rows,), device="cuda", dtype=torch.int32)
    ce = L.cross_entropy(7, id_type="i32")
    loss, lse, dx = run_ce(ce, rows, x, 8, t, "bf16")
    sub, tt = to_np(x[pick])[:, :7], t[pick].cpu().numpy()
    ref = O.cross_entropy(sub, tt)
    tol = ce_tol(sub, tt, 7, ref, 0.0, 0.0, 1.0, "bf16")
    within(loss[pick], ref[0], tol[0], "loss")
    within(dx[pick][:, :7], ref[2], tol[2], "dx")
    L.sppo_cross_entropy_bwd(ce, rows, x, 8, t, lse, None, dx, 8)
    within(dx[pick][:, :7], ref[2], tol[2] + 8 * U * np.abs(ref[1])[:, None], "dx from lse")


def test_cross_entropy_gradient_matches_differences():
    """Central differences of the fp32 loss: steps of 2^-4 have a third-order
    error of h^2/6 max|loss'''| (below 1, with z's 2 (3 z) added), and the two losses' roundings over
    2 h."""
    rows, V, h, z = 3, 50, 2.0 ** -4, 1e-2
    announce("cross entropy differences")
    x, t = ce_inputs(rows, V, 56, "f32", 2, scale=1.0)
    ce = L.cross_entropy(V, "f32", label_smoothing=0.2, z_loss=z)
    _, _, dx = run_ce(ce, rows, x.cuda(), 56, t.cuda(), "f32")
    for c in range(0, V, 7):
        up, down = x.clone(), x.clone()
        up[:, c] += h
        down[:, c] -= h
        f = [to_np(run_ce(ce, rows, v.cuda(), 56, t.cuda(), "f32", grad=False)[0]) for v in (up, down)]
        d = (f[0] - f[1]) / (to_np(up)[:, c] - to_np(down)[:, c])
        assert np.all(np.abs(d - to_np(dx)[:, c]) <= h * h / 6 * (1 + 60 * z) + 200 * U * 8 / h)


# -------------------------------------------------------------- gradient norm
def flat_views(sizes, dtype, shift=0, align=32, fill=0.0):
    """Views of one buffer, from multiples of `align` on, all `shift` further."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += -(-max(n, 1) // align) * align
    buf = torch.full((at + shift,), fill, dtype=dtype, device="cuda")
    return buf, [buf[shift + a:shift + a + n] for a, n in zip(places, sizes)]


RAGGED = [1, 7, 8, 9, 31, 32, 33, 0, 255, 2047, 2048, 2049, 4095, 4096, 4097, 12345]


@pytest.mark.parametrize("sizes,dtype,shift", [
    ([1], "f32", 0), (RAGGED, "f32", 0), (RAGGED, "bf16", 0), (RAGGED, "f32", 1), (RAGGED, "bf16", 1),
    ([3000001, 5], "bf16", 0), ([9 * 10 ** 6], "f32", 3),
])
def test_grad_norm(sizes, dtype, shift):
    announce(f"gradient norm {len(sizes)} tensors, {sum(sizes)} elements {dtype} shift={shift}")
    buf, views = flat_views(sizes, DT[dtype], shift, fill=1e30)  # what lies between is not read
    for i, v in enumerate(views):
        v.copy_(randn((len(v),), i, 10.0 ** (i % 5 - 2)).to(DT[dtype]))
    lst = L.opt_list([L.opt_tensor(len(v), grad=v, grad_dtype=dtype) for v in views], "none")
    n = L.sppo_grad_norm_workspace(lst)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    norm = np.sqrt(sum(float((to_np(v) ** 2).sum()) for v in views))
    steps = torch.tensor([41], device="cuda")
    for max_norm in (0.1 * norm, 3.0 * norm, INF):
        out = torch.full((2,), NAN, device="cuda")
        L.sppo_grad_norm(lst, max_norm, out, ws, n, steps)
        f = min(1.0, float(np.float32(max_norm)) / norm)
        within(out, [norm, f], 1.01 * U * np.array([norm, f]), "norm, factor")
    assert steps.item() == 44
    again = torch.empty_like(out)
    L.sppo_grad_norm(lst, INF, again, ws, n)
    assert torch.equal(again, out)


def test_grad_norm_of_extremes():
    announce("gradient norm of zeros, tiny, huge, infinite and NaN gradients")
    steps = torch.tensor([0], device="cuda")
    ws = torch.empty(2048 * 8, dtype=torch.uint8, device="cuda")
    out = torch.empty(2, device="cuda")
    # (value, norm of 100 of them, factor under 2, counted steps)
    for v, norm, f, count in ((0.0, 0.0, 1.0, 1), (1e-30, 1e-29, 1.0, 2), (1e30, 1e31, 2e-31, 3), (INF, INF, 0.0, 3),
                              (-INF, INF, 0.0, 3), (NAN, NAN, 0.0, 3), (3e38, INF, 0.0, 3)):
        g = torch.full((100,), v, device="cuda")
        lst = L.opt_list([L.opt_tensor(100, grad=g)], "none")
        L.sppo_grad_norm(lst, 2.0, out, ws, 2048 * 8, steps)
        within(out, np.array([norm, f]), 2 * U * np.nan_to_num(np.array([norm, f]), posinf=0.0) + 1e-45, v)
        assert steps.item() == count, v
    empty = L.opt_list([L.opt_tensor(0)], "none")
    L.sppo_grad_norm(empty, 2.0, out, ws, 2048 * 8)
    assert out.tolist() == [0.0, 1.0]


# ------------------------------------------------------------------------ AdamW
class Setting:
    """Tensors of an update in flat buffers, and their copies in NumPy."""

    def __init__(self, sizes, state, param, grad, shift=0, seed=0):
        self.sizes, self.state, self.param, self.grad = sizes, state, param, grad
        b = {}
        self.buf, self.v = b, {}

        def flat(name, dtype, fill=0.0):
            b[name], self.v[name] = flat_views(sizes, dtype, shift, fill=fill)

        flat("g", DT[grad], 3.0)
        flat("w", F32, 5.0)
        if param == "bf16":
            flat("p", BF, 5.0)
        small = state == "e4m3"
        for name in ("m", "v"):
            flat(name, torch.uint8 if small else F32)
            if small:
                b[name + "s"] = torch.zeros(len(b[name]) // 32 + 1, dtype=torch.uint8, device="cuda")
                at = np.cumsum([0] + [-(-max(n, 1) // 32) for n in sizes])
                self.v[name + "s"] = [b[name + "s"][a:a + -(-n // 32)] for a, n in zip(at, sizes)]
        for i, n in enumerate(sizes):
            self.v["w"][i].copy_(randn((n,), seed + 100 + i, 0.1))
            if param == "bf16":
                self.v["p"][i].copy_(self.v["w"][i])
        self.decay = [0.1 * (i % 3) for i in range(len(sizes))]
        self.lrs = [1.0 + 0.5 * (i % 2) for i in range(len(sizes))]
        ts = []
        for i, n in enumerate(sizes):
            kw = dict(grad=self.v["g"][i], grad_dtype=grad, m=self.v["m"][i], v=self.v["v"][i], param_dtype=param,
                      lr_scale=self.lrs[i], weight_decay=self.decay[i])
            kw.update(dict(param=self.v["p"][i], master=self.v["w"][i]) if param == "bf16" else
                      dict(param=self.v["w"][i]))
            if small:
                kw.update(m_scale=self.v["ms"][i], v_scale=self.v["vs"][i])
            ts.append(L.opt_tensor(n, **kw))
        self.list = L.opt_list(ts, state)

    def gradients(self, seed):
        for i, v in enumerate(self.v["g"]):
            v.copy_(randn((len(v),), seed + i, 10.0 ** (i % 4 - 3)))

    def np(self, name):
        return [t.cpu().numpy().copy() if t.dtype == torch.uint8 else to_np(t) for t in self.v[name]]

    def check_step(self, before, t, lr, b1, b2, eps, f, seed):
        """What a step made of `before`.  m: b1 m takes three roundings (b1, the
        product, the sum), (1 - b1) f g four: 4 u of both.  v: f g twice and four
        more: 6 u.  m / (1 - b1^t) / (sqrt ...): m's error, and 12 more
        roundings.  p: two of itself, four of what is taken off."""
        block0 = 0
        for i, n in enumerate(self.sizes):
            p, g, w = (to_np(before[k][i]) if not isinstance(before[k][i], np.ndarray) else before[k][i]
                       for k in ("w", "g", "w"))
            if self.state == "f32":
                m, v = before["m"][i], before["v"][i]
            else:
                m = O.value8(before["m"][i], before["ms"][i])
                r0 = O.value8(before["v"][i], before["vs"][i])
                v = r0 * r0
            lr_i, wd = lr * self.lrs[i], self.decay[i]
            rp, rm, rv = O.adamw(p, g, m, v, t, lr_i, b1, b2, eps, wd, f)
            tm = 4 * U * (np.abs(b1 * m) + (1 - b1) * np.abs(f * g)) + 2.0 ** -148
            tv = 6 * U * rv + 2.0 ** -148
            with np.errstate(all="ignore"):
                den = np.sqrt(rv / (1 - b2 ** t)) + eps
                q = rm / (1 - b1 ** t) / den
                tq = tm / (1 - b1 ** t) / den + 12 * U * np.abs(q)
            tp = abs(lr_i) * (tq + 4 * U * (np.abs(q) + np.abs(wd * p))) + 2 * U * np.abs(p)
            within(self.v["w"][i], rp, tp, ("w", i))
            if self.param == "bf16":
                assert torch.equal(self.v["p"][i], self.v["w"][i].to(BF)), ("param", i)
            if self.state == "f32":
                within(self.v["m"][i], rm, tm, ("m", i))
                within(self.v["v"][i], rv, tv, ("v", i))
            else:
                self.check_codes(i, n, m, v, g, b1, b2, f, t, seed, block0)
            block0 += -(-n // 32)

    def check_codes(self, i, n, m, v, g, b1, b2, f, t, seed, block0):
        """The states that are rounded are IEEE results of single operations, so
        NumPy's fp32 has the same ones; the codes are those of the oracle's
        rounding of them but where a draw falls within 2^-20 of its threshold
        (values below 2^-6 lose bits below 2^-29 when 2^-6 is added)."""
        s = np.float32
        fg = g.astype(s) * s(f)
        m32 = s(b1) * m.astype(s) + s(1 - b1) * fg
        v32 = s(b2) * v.astype(s) + s(1 - b2) * (fg * fg)
        u = O.draws(n, block0, t, seed)
        for name, x, bits in (("m", m32, u & np.uint64(0xFFFF)), ("v", np.sqrt(v32), u >> np.uint64(16))):
            scales = O.block_bytes(x)
            got = self.v[name + "s"][i].cpu().numpy()
            assert np.array_equal(got, scales), (name, i, np.argwhere(got != scales)[:3])
            codes, far = O.round8(x, scales, bits.astype(np.float64), name == "v")
            have = self.v[name][i].cpu().numpy()
            bad = (have != codes) & (far > 2.0 ** -20)
            assert not bad.any(), (name, i, np.argwhere(bad)[:3].tolist(), have[bad][:3], codes[bad][:3], x[bad][:3])


COMBOS = [("f32", "f32", "f32", 0), ("f32", "bf16", "f32", 0), ("f32", "f32", "bf16", 0), ("f32", "bf16", "bf16", 0),
          ("f32", "bf16", "f32", 1), ("f32", "f32", "bf16", 1), ("e4m3", "bf16", "bf16", 0), ("e4m3", "f32", "f32", 0),
          ("e4m3", "bf16", "f32", 0), ("e4m3", "f32", "bf16", 0)]


@pytest.mark.parametrize("state,param,grad,shift", COMBOS)
@pytest.mark.parametrize("sizes", [[1], RAGGED, [70001, 64, 4096 * 3]])
def test_adamw(state, param, grad, shift, sizes):
    """Three steps from zero states, each against the oracle from what the step
    before left; what lies between the tensors stays."""
    announce(f"adamw {state} param={param} grad={grad} shift={shift} sizes={sizes}")
    k = Setting(sizes, state, param, grad, shift)
    lr, b1, b2, eps, seed = 1e-2, 0.9, 0.99, 1e-8, 2 ** 50 + 3
    norm = torch.tensor([3.0, 0.7], device="cuda")
    f = float(norm[1])
    names = ["w", "g", "m", "v"] + (["ms", "vs"] if state == "e4m3" else [])
    inside = {n: torch.zeros(b.shape, dtype=torch.bool, device="cuda") for n, b in k.buf.items()}
    for n, views in k.v.items():
        for t in views:
            inside[n][t.storage_offset():t.storage_offset() + len(t)] = True
    outside = {n: b[~inside[n]].clone() for n, b in k.buf.items()}
    for t in (1, 2, 2 ** 33 + 5):
        k.gradients(7 * t % 1000)
        before = {n: k.np(n) for n in names}
        L.sppo_adamw_step(k.list, L.adamw(lr, b1, b2, eps, t, norm=norm, seed=seed))
        k.check_step(before, t, lr, b1, b2, eps, f, seed)
    for n, b in k.buf.items():
        assert torch.equal(b[~inside[n]], outside[n]), n


def test_adamw_counts_and_schedules_on_the_device():
    """step_dev and lr_dev against the same numbers from the host: the same bits."""
    announce("adamw step and lr on the device")
    a, b = (Setting(RAGGED, "f32", "bf16", "f32") for _ in range(2))
    for k in (a, b):
        k.gradients(3)
    L.sppo_adamw_step(a.list, L.adamw(1e-2, step=1234))
    step, lr = torch.tensor([1200], device="cuda"), torch.tensor([1e-2], device="cuda")
    L.sppo_adamw_step(b.list, L.adamw(1.0, step=34, step_dev=step, lr_dev=lr))
    for n in a.buf:
        assert torch.equal(a.buf[n], b.buf[n]), n
    # Below one counts as one.
    step.fill_(-50)
    L.sppo_adamw_step(b.list, L.adamw(1e-2, step=0, step_dev=step))
    L.sppo_adamw_step(a.list, L.adamw(1e-2, step=1))
    for n in a.buf:
        assert torch.equal(a.buf[n], b.buf[n]), n


def test_an_update_past_32_bit_offsets():
    """One tensor of 2^32 + 37 elements: the norm of gradients at its ends, and the
    update there."""
    announce("update past 2^32 elements")
    n = 2 ** 32 + 37
    g = torch.zeros(n, dtype=BF, device="cuda")
    w = torch.ones(n, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(n // 32 + 1, dtype=torch.uint8, device="cuda") for _ in range(2))
    ends = torch.tensor([0, 5, 2 ** 32 - 1, 2 ** 32, n - 3, n - 1], device="cuda")
    g[ends] = torch.tensor([1.0, -2.0, 3.0, -4.0, 5.0, -6.0], device="cuda", dtype=BF)
    lst = L.opt_list([L.opt_tensor(n, g, "bf16", w, "f32", None, m, v, ms, vs)], "e4m3")
    out = torch.empty(2, device="cuda")
    ws = torch.empty(L.sppo_grad_norm_workspace(lst), dtype=torch.uint8, device="cuda")
    L.sppo_grad_norm(lst, INF, out, ws, ws.numel())
    assert abs(out[0].item() - 91 ** 0.5) <= U * 91 ** 0.5 * 1.01
    L.sppo_adamw_step(lst, L.adamw(0.5, 0.9, 0.99, 1e-8, 1))
    # The first step goes lr against the gradient's sign: 16 roundings of one, and eps / |g|.
    assert torch.all((w[ends] - 1.0 + 0.5 * torch.sign(g[ends].float())).abs() <= 16 * U + 1e-8)
    w[ends] = 1.0
    assert torch.all(w == 1.0) and int((m != 0).sum()) == len(ends) and int((v != 0).sum()) == len(ends)


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_adamw_leaves_all_as_it_is_without_a_norm(state):
    announce(f"adamw {state} under an infinite norm")
    k = Setting(RAGGED, state, "bf16", "f32")
    k.gradients(1)
    L.sppo_adamw_step(k.list, L.adamw(1e-2))
    before = {n: b.clone() for n, b in k.buf.items()}
    k.v["g"][4][3] = NAN
    before["g"] = k.buf["g"].clone()
    for bad in (INF, NAN):
        norm = torch.tensor([bad, 0.0], device="cuda")
        L.sppo_adamw_step(k.list, L.adamw(1e-2, norm=norm))
        for n, b in k.buf.items():
            assert torch.equal(b.view(torch.uint8), before[n].view(torch.uint8)), n


def test_adamw_of_extreme_gradients():
    """Zeros, infinities and NaN among fp32 and 8-bit states: their own elements
    only."""
    announce("adamw of extreme gradients")
    for state in ("f32", "e4m3"):
        k = Setting([96], state, "f32", "f32")
        g = k.v["g"][0]
        g.fill_(0.0)
        g[40], g[41], g[70] = INF, NAN, 1e-3
        w0 = k.v["w"][0].clone()
        L.sppo_adamw_step(k.list, L.adamw(1e-2, 0.9, 0.99, 1e-8, 1))
        w = k.v["w"][0]
        assert torch.isnan(w[[40, 41]]).all()
        rest = [i for i in range(96) if i not in (40, 41, 70)]
        assert torch.equal(w[rest], w0[rest]) and abs((w0[70] - w[70]).item() - 1e-2) < 1e-6
        if state == "e4m3":
            m, v = (O.value8(k.v[n][0].cpu().numpy(), k.v[n + "s"][0].cpu().numpy()) for n in ("m", "v"))
            assert np.isnan(m[[40, 41]]).all() and np.isnan(v[[40, 41]]).all()
            assert not m[rest].any() and not v[rest].any()


@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("f", [1.0, 0.5])
def test_adamw_of_gradients_whose_squares_are_infinite(param, f):
    """Finite gradients from 1.8e19 on, whose squares leave fp32's range, beside
    small ones.  With 8-bit states three steps against the oracle, each from what
    the one before left: parameters as check_step counts them, states to a step
    of their codes (2^-3 of a value, 2^-9 of the block's unit at least).  With
    fp32 states v is infinite and the parameter only decays."""
    announce(f"adamw of gradients with infinite squares param={param} f={f}")
    lr, b1, b2, eps = 1e-2, 0.9, 0.99, 1e-8
    norm = torch.tensor([3.0, f], device="cuda")
    big = [1.7e19, 1.9e19, -2e19, 1e25, -3e30, 1e38, -3.3e38]
    k = Setting([133, 96], "e4m3", param, "f32")
    for t in (1, 2, 3):
        k.gradients(t)
        for i, v in enumerate(big):
            k.v["g"][0][3 + 7 * i + 40 * (i % 2)] = v if t != 2 else 1e-3
            k.v["g"][1][95 - i] = v
        before = {n: k.np(n) for n in ("w", "g", "m", "v", "ms", "vs")}
        L.sppo_adamw_step(k.list, L.adamw(lr, b1, b2, eps, t, norm=norm, seed=11))
        for i, n in enumerate(k.sizes):
            w, g = before["w"][i], before["g"][i]
            m, r = (O.value8(before[a][i], before[a + "s"][i]) for a in ("m", "v"))
            rp, rm, rv = O.adamw(w, g, m, r * r, t, lr * k.lrs[i], b1, b2, eps, k.decay[i], f)
            rr = np.sqrt(rv)
            tm = 4 * U * (np.abs(b1 * m) + (1 - b1) * np.abs(f * g)) + 2.0 ** -148
            den = rr / np.sqrt(1 - b2 ** t) + eps
            q = rm / (1 - b1 ** t) / den
            tq = tm / (1 - b1 ** t) / den + 12 * U * np.abs(q)
            tp = lr * k.lrs[i] * (tq + 4 * U * (np.abs(q) + np.abs(k.decay[i] * w))) + 2 * U * np.abs(w)
            within(k.v["w"][i], rp, tp, ("w", t, i))
            for a, x in (("m", rm), ("v", rr)):
                scales = k.v[a + "s"][i].cpu().numpy()
                assert np.array_equal(scales, O.block_bytes(x)), (a, t, i)
                unit = 2.0 ** (np.repeat(scales.astype(np.float64), 32)[:n] - 127)
                got = torch.from_numpy(O.value8(k.v[a][i].cpu().numpy(), scales))
                within(got, x, 2.0 ** -3 * np.abs(x) + 2.0 ** -9 * unit, (a, t, i))
    k = Setting([96], "f32", param, "f32")
    k.gradients(1)
    k.v["g"][0][5], k.v["g"][0][64] = 1e25, -3.3e38
    w0 = k.np("w")[0]
    L.sppo_adamw_step(k.list, L.adamw(lr, b1, b2, eps, 1, norm=norm))
    assert torch.isinf(k.v["v"][0][[5, 64]]).all() and torch.isfinite(k.v["w"][0]).all()
    within(k.v["w"][0][[5, 64]], w0[[5, 64]], 0.0, "w under an infinite v")


@pytest.mark.parametrize("b1,b2", [(0.0, 0.99), (0.9, 0.0), (0.0, 0.0)])
def test_adamw_states_at_the_end_of_the_range(b1, b2):
    """With a beta of zero a state is as large as its gradient: rounding up must
    not make 256 2^120, which is past fp32's range, of 8-bit states.  Three steps
    under large gradients, and with beta1 zero one under small ones (else m over a
    small r is itself past the range), leave finite parameters, each step within
    check_step's count of roundings, and states to a step of their codes (2^-3)."""
    announce(f"adamw states at the end of the range betas={b1},{b2}")
    lr, eps = 1e-2, 1e-8
    k = Setting([256], "e4m3", "f32", "f32")
    for t in (1, 2, 3, 4) if b1 == 0.0 else (1, 2, 3):
        k.gradients(t)
        if t < 4:
            big = torch.linspace(3.1e38, 3.4e38, 200, device="cuda")
            k.v["g"][0][20:220] = torch.where(torch.arange(200, device="cuda") % 3 == t % 3, -big, big)
        w, g = k.np("w")[0], k.np("g")[0]
        m, r = (O.value8(k.np(a)[0], k.np(a + "s")[0]) for a in ("m", "v"))
        assert np.abs(m).max() < 2.0 ** 128 and r.max() < 2.0 ** 128
        L.sppo_adamw_step(k.list, L.adamw(lr, b1, b2, eps, t, seed=t))
        rp, rm, rv = O.adamw(w, g, m, r * r, t, lr * k.lrs[0], b1, b2, eps, k.decay[0])
        tm = 4 * U * (np.abs(b1 * m) + (1 - b1) * np.abs(g)) + 2.0 ** -148
        den = np.sqrt(rv / (1 - b2 ** t)) + eps
        q = rm / (1 - b1 ** t) / den
        tp = lr * k.lrs[0] * (tm / (1 - b1 ** t) / den + 16 * U * np.abs(q)) + 2 * U * np.abs(w)
        within(k.v["w"][0], rp, tp, ("w", t))
        for a, x in (("m", rm), ("v", np.sqrt(rv))):
            scales = k.v[a + "s"][0].cpu().numpy()
            unit = 2.0 ** (np.repeat(scales.astype(np.float64), 32)[:256] - 127)
            got = O.value8(k.v[a][0].cpu().numpy(), scales)
            assert np.all(np.abs(got - x) <= 2.0 ** -3 * np.abs(x) + 2.0 ** -9 * unit), (a, t)


# --------------------------------------------------------------------- together
def test_a_step_in_graphs():
    """Rotary, loss, norm and update captured twice with their own buffers and
    replayed on two streams with eager work between: every replay has the eager
    call's bits, and the count of steps goes on."""
    announce("step operators in two graphs")
    rows, V, h, D = 65, 5003, 4, 64
    ld = 5008

    def work(seed):
        freqs, dev, amp = table(D)
        x = randn((rows, ld), seed, 2.0).to(BF).cuda()
        t = torch.randint(-1, V, (rows,), generator=torch.Generator().manual_seed(seed)).cuda()
        q = randn((rows, h * D), seed + 1).to(BF).cuda()
        k = Setting([5000, 33, 7], "e4m3", "bf16", "f32", seed=seed)
        k.gradients(seed)
        ce = L.cross_entropy(V, scale=1.0 / rows)
        ws, n = workspace(ce, rows)
        nws = torch.empty(L.sppo_grad_norm_workspace(k.list), dtype=torch.uint8, device="cuda")
        s = dict(loss=torch.empty(rows, device="cuda"), dx=torch.zeros_like(x), y=torch.empty_like(q),
                 norm=torch.empty(2, device="cuda"), steps=torch.zeros(1, dtype=torch.int64, device="cuda"), k=k)

        def call():
            L.sppo_rotary_apply(L.rotary(D, dev, "half", amp, 100), rows,
                                L.rotary_tensors([L.rotary_tensor(h, D, q, h * D, D, s["y"], h * D, D)]))
            L.sppo_cross_entropy(ce, rows, x, ld, t, s["loss"], None, s["dx"], ld, ws, n)
            L.sppo_grad_norm(k.list, 0.5, s["norm"], nws, nws.numel(), s["steps"])
            L.sppo_adamw_step(k.list, L.adamw(1e-2, step=0, step_dev=s["steps"], norm=s["norm"], seed=seed))

        s["keep"] = (dev, x, t, q, ws, nws)
        return call, s

    def state(s):
        return [s[n].clone() for n in ("loss", "dx", "y", "norm", "steps")] + [b.clone() for b in s["k"].buf.values()]

    eager, graphs = [], []
    for seed in (1, 2):
        call, s = work(seed)
        runs = []
        for _ in range(4):
            call()
            runs.append(state(s))
        eager.append(runs)
        call, s = work(seed)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call()
        graphs.append((g, stream, s))
    torch.cuda.synchronize()
    for r in range(4):
        for g, stream, s in graphs:
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        (torch.randn(1000, device="cuda") * 2).sum().item()
        for (g, stream, s), runs in zip(graphs, eager):
            for a, b in zip(state(s), runs[r]):
                assert torch.equal(a, b)
    assert graphs[0][2]["steps"].item() == 4
