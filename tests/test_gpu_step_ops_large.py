"""The operators that close a training step at sizes that take other paths than
small ones: tensors of 32 MiB and more, which go past the caches, logits in more
slices than one, and what lies on both sides of a border between kernels.

A row's arithmetic does not depend on how many rows a call has, so large calls
have the bits of the same rows in small ones; rows here and there, and updates,
are held against the fp64 oracle with the tolerances of test_gpu_step_ops.py.
"""
import numpy as np
import pytest
import torch

from oracle import step_ops as O
from paper_2503_10377_amd import sppo as L
from parity import to_np
from test_gpu_step_ops import (BF, DT, INF, U, Setting, announce, ce_tol, flat_views, rotary_check, run_ce, table,
                               within)

pytestmark = pytest.mark.gpu


def noise(shape, seed, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(DT[dtype])


# ------------------------------------------------------------------- rotary
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot,dtype", [(128, 128, "bf16"), (128, 48, "bf16"), (72, 24, "bf16"), (128, 64, "f32")])
def test_rotary_of_large_tensors(D, rot, dtype, layout):
    """32 MiB and more in one call, out of place and in place, against the same
    rows in calls of less."""
    h = 16
    rows = 2 ** 25 // (h * D * DT[dtype].itemsize) + 5
    announce(f"rotary of large tensors rows={rows} D={D} rot={rot} {layout} {dtype}")
    freqs, dev, amp = table(rot)
    x = noise((rows, h * D), 1, dtype)
    few = noise((rows, 2 * D), 2, "f32")

    def turn(a, b, c0, c1, inverse=0):
        ts = [L.rotary_tensor(n, D, s[c0:c1], n * D, D, d[c0:c1], n * D, D, dt)
              for (s, d), n, dt in ((a, h, dtype), (b, 2, "f32"))]
        L.sppo_rotary_apply(L.rotary(rot, dev, layout, amp, 77 + c0), c1 - c0, L.rotary_tensors(ts), inverse)

    whole, whole2 = torch.empty_like(x), torch.empty_like(few)
    turn((x, whole), (few, whole2), 0, rows)
    parts, parts2 = torch.empty_like(x), torch.empty_like(few)
    for c0, c1 in ((0, 7), (7, rows // 2), (rows // 2, rows)):
        turn((x, parts), (few, parts2), c0, c1)
    assert torch.equal(whole, parts) and torch.equal(whole2, parts2)
    pick = [0, 1, rows // 2, rows - 1]
    for y, s, n, dt in ((whole, x, h, dtype), (whole2, few, 2, "f32")):
        rotary_check(y[pick].reshape(-1, n, D), s[pick].reshape(-1, n, D), [77 + r for r in pick], freqs, rot, layout,
                     amp, 0, dt, "y")
    turn((x, x), (few, few), 0, rows)
    assert torch.equal(whole, x) and torch.equal(whole2, few)


# --------------------------------------------------------------------- loss
def ce_case(rows, V, ld, dtype, buf=None):
    """Logits [rows, ld] and targets, every fifth row without one."""
    x = noise((rows, ld), V, dtype, 3.0)
    if buf is not None:
        buf[:, :ld] = x
    t = torch.randint(0, V, (rows,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    t[1::5] = V
    return x, t


def ce_rows(ce, x, ld, t, pieces, lse=None, dloss=None):
    """Loss, lse and gradient (or the gradient from lse) in calls of those rows."""
    out = []
    for c0, c1 in pieces:
        if lse is None:
            out.append(run_ce(ce, c1 - c0, x[c0:c1], ld, t[c0:c1], "bf16" if x.dtype == BF else "f32"))
        else:
            dx = torch.full_like(x[c0:c1], 7.0)
            L.sppo_cross_entropy_bwd(ce, c1 - c0, x[c0:c1], ld, t[c0:c1], lse[c0:c1], dloss[c0:c1], dx, ld)
            out.append((dx,))
    return [torch.cat(v) for v in zip(*out)]


# (rows, V, dtype, the largest small call's rows): of rows in registers in teams
# of 64, 256, 512 and 1024 threads; in parts; in parts and two slices of 160 MiB
# (639 rows a slice of 131081 bf16 or 65601 fp32 logits).
@pytest.mark.parametrize("rows,V,dtype,step", [
    (70000, 250, "bf16", 30000), (40000, 509, "f32", 9000), (3000, 8191, "bf16", 1500), (1100, 8191, "f32", 700),
    (300, 33001, "f32", 150), (140, 65535, "f32", 128), (140, 65601, "f32", 50), (140, 131081, "bf16", 50),
    (700, 131081, "bf16", 100), (700, 65601, "f32", 100),
])
def test_cross_entropy_of_large_logits(rows, V, dtype, step):
    announce(f"cross entropy of large logits rows={rows} V={V} {dtype}")
    ld = (V + 7) // 8 * 8 + 8
    x, t = ce_case(rows, V, ld, dtype)
    ce = L.cross_entropy(V, dtype, label_smoothing=0.1, z_loss=1e-3, scale=0.5)
    pieces = [(c, min(c + step, rows)) for c in range(0, rows, step)]
    if step == 128:  # rows of this length are kept in registers from 128 of them on
        pieces = [(0, 128), (12, 140)]
    whole = ce_rows(ce, x, ld, t, [(0, rows)])
    small = ce_rows(ce, x, ld, t, pieces)
    if step == 128:
        small = [torch.cat([s[:128], s[244:]]) for s in small]
    for a, b, what in zip(whole, small, ("loss", "lse", "dx")):
        assert torch.equal(a, b), what
    loss, lse, dx = whole
    assert torch.all(dx[:, V:] == 7.0), "columns past V written"
    per = 160 * 2 ** 20 // (V * DT[dtype].itemsize)
    pick = sorted({0, 1, 2, min(per, rows) - 1, min(per, rows - 1), min(per + 1, rows - 1), rows - 2, rows - 1})
    sub, tt = to_np(x[pick])[:, :V], t[pick].cpu().numpy()
    ref = O.cross_entropy(sub, tt, 0.1, 1e-3, 0.5)
    tol = ce_tol(sub, tt, V, ref, 0.1, 1e-3, 0.5, dtype)
    for got, r, e, what in zip((loss[pick], lse[pick], dx[pick][:, :V]), ref, tol, ("loss", "lse", "dx")):
        within(got, r, e, what)
    dloss = noise((rows,), 8, "f32")
    back = ce_rows(ce, x, ld, t, [(0, rows)], lse, dloss)[0]
    for c0, c1 in [(0, step), (rows - step, rows)]:
        assert torch.equal(back[c0:c1], ce_rows(ce, x, ld, t, [(c0, c1)], lse, dloss)[0])
    ref = O.cross_entropy(sub, tt, 0.1, 1e-3, 0.5, to_np(lse[pick]), to_np(dloss[pick]))
    tol = ce_tol(sub, tt, V, ref, 0.1, 1e-3, 0.5, dtype, to_np(lse[pick]), to_np(dloss[pick]))
    within(back[pick][:, :V], ref[2], tol[2], "dx from lse")
    tail = x[:, V:].clone()
    over = run_ce(ce, rows, x, ld, t, dtype, in_place=True)
    for a, b, what in zip(over[:2], whole[:2], ("loss", "lse")):
        assert torch.equal(a, b), what
    assert torch.equal(x[:, :V], dx[:, :V]) and torch.equal(x[:, V:], tail)


@pytest.mark.parametrize("V,dtype", [(32768, "bf16"), (32769, "bf16"), (40001, "bf16"), (40001, "f32"),
                                     (131072, "bf16"), (131073, "bf16"), (65536, "f32"), (65537, "f32")])
@pytest.mark.parametrize("rows", [1, 127, 128])
def test_cross_entropy_around_the_borders(V, dtype, rows):
    """Few long rows go in parts, from 128 rows or up to 32768 logits in one piece;
    above 131072 bf16 or 65536 fp32 all do.  In place, and the loss alone, too."""
    announce(f"cross entropy around the borders rows={rows} V={V} {dtype}")
    ld = (V + 7) // 8 * 8
    x, t = ce_case(rows, V, ld, dtype)
    ce = L.cross_entropy(V, dtype, scale=2.0)
    loss, lse, dx = run_ce(ce, rows, x, ld, t, dtype)
    pick = sorted({0, min(1, rows - 1), rows - 1})
    sub, tt = to_np(x[pick])[:, :V], t[pick].cpu().numpy()
    ref = O.cross_entropy(sub, tt, scale=2.0)
    tol = ce_tol(sub, tt, V, ref, 0.0, 0.0, 2.0, dtype)
    for got, r, e, what in zip((loss[pick], lse[pick], dx[pick][:, :V]), ref, tol, ("loss", "lse", "dx")):
        within(got, r, e, what)
    alone = run_ce(ce, rows, x, ld, t, dtype, grad=False)
    over = run_ce(ce, rows, x, ld, t, dtype, in_place=True)
    for r in (alone, over):
        assert torch.equal(r[0], loss) and torch.equal(r[1], lse)
    assert torch.equal(x[:, :V], dx[:, :V])


@pytest.mark.parametrize("rows,V,dtype", [(128, 40001, "bf16"), (200, 65536, "f32"), (5, 32768, "bf16")])
def test_cross_entropy_without_the_workspace_that_it_does_not_use(rows, V, dtype):
    """NULL where rows are kept in registers: the bits of a call that has one."""
    announce(f"cross entropy without a workspace rows={rows} V={V} {dtype}")
    ld = (V + 7) // 8 * 8
    x, t = ce_case(rows, V, ld, dtype)
    ce = L.cross_entropy(V, dtype)
    want = run_ce(ce, rows, x, ld, t, dtype)
    loss, lse, dx = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.full_like(want[2], 7.0)
    L.sppo_cross_entropy(ce, rows, x, ld, t, loss, lse, dx, ld)
    for a, b in zip((loss, lse, dx), want):
        assert torch.equal(a, b)


def test_cross_entropy_in_parts_past_32_bit_offsets():
    """Rows in parts whose offsets pass 2^32 elements, in place, in a buffer that
    is touched at few places."""
    announce("cross entropy in parts past 2^32 elements")
    rows, V, ld = 70, 131081, 1 << 26
    buf = torch.empty(rows * ld, dtype=BF, device="cuda").view(rows, ld)
    x, t = ce_case(rows, V, V + 7, "bf16", buf)
    assert (V + 7) % 8 == 0
    ce = L.cross_entropy(V)
    want = run_ce(ce, rows, x, V + 7, t, "bf16")
    got = run_ce(ce, rows, buf, ld, t, "bf16", in_place=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(buf[:, :V], want[2][:, :V]) and torch.equal(buf[:, V:V + 7], x[:, V:])
    buf[:, :V + 7] = x
    L.sppo_cross_entropy_bwd(ce, rows, buf, ld, t, want[1], None, buf, ld)
    back = torch.empty_like(x)
    L.sppo_cross_entropy_bwd(ce, rows, x, V + 7, t, want[1], None, back, V + 7)
    assert torch.equal(buf[:, :V], back[:, :V]) and torch.equal(buf[:, V:V + 7], x[:, V:])
    sub, tt = to_np(x[-2:])[:, :V], t[-2:].cpu().numpy()
    ref = O.cross_entropy(sub, tt)
    tol = ce_tol(sub, tt, V, ref, 0.0, 0.0, 1.0, "bf16")
    within(want[0][-2:], ref[0], tol[0], "loss")
    within(want[2][-2:, :V], ref[2], tol[2], "dx")


# --------------------------------------------------------------------- update
@pytest.mark.parametrize("state,param,grad,shift", [("f32", "bf16", "f32", 0), ("f32", "f32", "bf16", 1),
                                                    ("f32", "bf16", "bf16", 1), ("e4m3", "bf16", "f32", 0),
                                                    ("e4m3", "f32", "bf16", 0)])
def test_adamw_of_a_large_list(state, param, grad, shift):
    """Lists of 2^23 elements and more go past the caches: two steps, each against
    the oracle from what the step before left."""
    announce(f"adamw of a large list {state} param={param} grad={grad} shift={shift}")
    k = Setting([2 ** 23 - 4000, 70001, 33, 4097], state, param, grad, shift)
    names = ["w", "g", "m", "v"] + (["ms", "vs"] if state == "e4m3" else [])
    norm = torch.tensor([3.0, 0.7], device="cuda")
    for t in (1, 2):
        k.gradients(7 * t)
        before = {n: k.np(n) for n in names}
        L.sppo_adamw_step(k.list, L.adamw(1e-2, 0.9, 0.99, 1e-8, t, norm=norm, seed=5))
        k.check_step(before, t, 1e-2, 0.9, 0.99, 1e-8, float(norm[1]), 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grad_norm_of_a_large_list(dtype):
    """More tiles than workgroups, several a workgroup, past the caches."""
    announce(f"gradient norm of a large list {dtype}")
    _, views = flat_views([2 ** 23 + 5, 4 * 10 ** 6, 77], DT[dtype], 1, fill=1e30)
    for i, v in enumerate(views):
        v.copy_(noise((len(v),), i, dtype))
    lst = L.opt_list([L.opt_tensor(len(v), grad=v, grad_dtype=dtype) for v in views], "none")
    n = L.sppo_grad_norm_workspace(lst)
    ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(2, device="cuda")
    want = sum(float((to_np(v) ** 2).sum()) for v in views) ** 0.5
    L.sppo_grad_norm(lst, 0.5 * want, out, ws, n)
    within(out, [want, float(np.float32(0.5 * want)) / want], 1.01 * U * np.array([want, 0.5]), "norm, factor")
    again = torch.empty_like(out)
    L.sppo_grad_norm(lst, INF, again, ws, n)
    assert again[0] == out[0] and again[1] == 1.0
