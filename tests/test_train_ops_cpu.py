"""The training operators without a GPU: the oracle's pins (the generator's
published answers, central differences of every gradient), and what the
library refuses before it touches a device."""
import ctypes

import numpy as np
import pytest

from oracle import train_ops as O
from paper_2503_10377_amd import sppo as L

BAD, UNSUP = L.SPPO_ERR_INVALID_ARG, L.SPPO_ERR_UNSUPPORTED


# ------------------------------------------------------------------ the oracle
@pytest.mark.parametrize("counter,key,answer", [
    # the known answers that the generator's authors publish for Philox4x32-10
    ([0, 0, 0, 0], [0, 0], [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
     [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]),
])
def test_philox_known_answers(counter, key, answer):
    assert [int(v) for v in O.philox4x32(np.array(counter, dtype=np.uint64), key)] == answer


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
def test_kept_share_and_scale(p):
    """The kept share over N draws lies within 5 standard deviations of the
    drawn probability, and its inverse is the scale."""
    rows, W = 500, 512
    k = O.keep_factor(rows, W, p, seed=77, offset=3)
    q = 1.0 - O.threshold(p) / 65536.0
    assert abs((k > 0).mean() - q) <= 5 * np.sqrt(q * (1 - q) / (rows * W))
    assert np.all((k == 0) | (k == 1 / q))


def test_mask_depends_on_the_global_position_only():
    a = O.keep_factor(40, 64, 0.3, seed=5, offset=9, row0=100)
    b = O.keep_factor(15, 64, 0.3, seed=5, offset=9, row0=117)
    assert np.array_equal(a[17:32], b)
    assert not np.array_equal(a, O.keep_factor(40, 64, 0.3, seed=5, offset=10, row0=100))
    assert not np.array_equal(a, O.keep_factor(40, 64, 0.3, seed=6, offset=9, row0=100))


CONFIGS = [("layer", "layer", "channel", True), ("rms", "rms", "token", False), ("none", "layer", "none", True),
           ("layer", "none", "token", True), ("none", "rms", "channel", True), ("rms", "layer", "channel", True),
           ("none", "none", "token", False)]


@pytest.mark.parametrize("post,pre,gate,beta", CONFIGS)
def test_block_norm_gradients_match_differences(post, pre, gate, beta):
    """Central differences (step e = 1e-5) of sum(dz z) + sum(dh h): their
    error is e^2 / 6 times a third derivative of order 10 at these sizes
    (2e-10) and the rounding of a sum of 160 terms of order 1 over 2 e
    (160 * 1.1e-16 / 2e-5 = 1e-9); gate 1e-7."""
    g = np.random.default_rng(3)
    rows, W = 5, 16
    cfg = dict(post=post, pre=pre, gate=gate, eps=1e-5, alpha=0.8, scale=0.7)
    arr = {"x": g.normal(size=(rows, W)), "b": g.normal(size=(rows, W)) * 2 + 0.5}
    if post != "none":
        arr["post_gamma"] = 1 + 0.2 * g.normal(size=W)
    if pre != "none":
        arr["pre_gamma"] = 1 + 0.2 * g.normal(size=W)
    for k in ("post", "pre"):
        if beta and k + "_gamma" in arr:
            arr[k + "_beta"] = 0.3 * g.normal(size=W)
    if gate != "none":
        arr["gate"] = g.uniform(0.5, 1.5, size=W if gate == "channel" else rows)
    keep = O.keep_factor(rows, W, 0.25, seed=1, offset=2, row0=3)
    dz, dh = g.normal(size=(rows, W)), g.normal(size=(rows, W))

    def loss(a):
        f = O.block_norm_fwd(a["x"], a["b"], cfg, a, keep)
        return (dh * f["h"]).sum() + ((dz * f["z"]).sum() if pre != "none" else 0.0)

    f = O.block_norm_fwd(arr["x"], arr["b"], cfg, arr, keep)
    grad = O.block_norm_bwd(arr["b"], f["h"], f, dz, dh, cfg, arr, keep)
    names = {"x": "dx", "b": "db"}
    for name, v in arr.items():
        got = grad[names.get(name, name)]
        for idx in np.ndindex(v.shape):
            e = 1e-5
            up, dn = dict(arr), dict(arr)
            up[name], dn[name] = v.copy(), v.copy()
            up[name][idx] += e
            dn[name][idx] -= e
            assert abs((loss(up) - loss(dn)) / (2 * e) - got[idx]) <= 1e-7, (name, idx)


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    """sum(dy y) = sum(dtable table): both sides are the same products, of
    order 1, 640 of them, summed in another order (gate 640 * 2^-53 * 10)."""
    g = np.random.default_rng(4)
    V, W, rows = 7, 16, 40
    ids = g.integers(-2, V + 2, size=rows)
    table, dy = g.normal(size=(V, W)), g.normal(size=(rows, W))
    keep = O.keep_factor(rows, W, 0.2, seed=8)
    lhs = (dy * O.embedding_fwd(ids, table, 3.0, keep)).sum()
    rhs = (O.embedding_bwd(ids, dy, V, 3.0, keep) * table).sum()
    assert abs(lhs - rhs) <= 640 * 2.0 ** -53 * 10 * 10


@pytest.mark.parametrize("norm,gate", [("layer", True), ("rms", False), ("none", False), ("none", True)])
def test_layer_with_ends_matches_differences(norm, gate):
    """Central differences (step 1e-5) of L = sum(dy y) along one random
    direction of every input and parameter: rounding 1e3 terms of order 1 times
    1.1e-16 / 2e-5 = 6e-9, truncation 1e-10 times a third derivative along the
    direction of order 1e3; gate 1e-6 of the sum of magnitudes."""
    g = np.random.default_rng(11)
    S, hq, hkv, d = 6, 2, 1, 4
    H = hq * d
    p = {"w_qkv": g.normal(size=(H, (hq + 2 * hkv) * d)) / 3, "w_o": g.normal(size=(H, H)) / 3,
         "w_1": g.normal(size=(H, 4 * H)) / 3, "w_2": g.normal(size=(4 * H, H)) / 6,
         "g1": 1 + 0.1 * g.normal(size=H), "b1": 0.1 * g.normal(size=H),
         "g2": 1 + 0.1 * g.normal(size=H), "b2": 0.1 * g.normal(size=H)}
    for n in (1, 2):
        if norm != "none":
            p[f"g_end{n}"] = 1 + 0.1 * g.normal(size=H)
        if norm == "layer":
            p[f"b_end{n}"] = 0.1 * g.normal(size=H)
        if gate:
            p[f"gate{n}"] = g.uniform(0.5, 1.5, size=H)
    ends = dict(norm=norm, gate=gate, alpha=0.9, scale=0.7)
    keep = [O.keep_factor(S, H, 0.25, 5, o) for o in (1, 2)]
    x, dy = g.normal(size=(S, H)), g.normal(size=(S, H))
    run = lambda q: O.layer_with_ends(q["x"], dy, q, hq, hkv, d, ends, *keep)
    base = dict(p, x=x)
    ref = run(base)
    assert set(ref) == {"y"} | {"d" + k for k in base}
    for name, val in base.items():
        t = g.normal(size=val.shape)
        up, dn = (run(dict(base, **{name: val + s * 1e-5 * t})) for s in (1, -1))
        diff = (dy * (up["y"] - dn["y"])).sum() / 2e-5
        along = ref["d" + name] * t
        assert abs(diff - along.sum()) <= 1e-6 * np.abs(along).sum() + 1e-8, name


def test_layer_with_plain_ends_is_the_layer():
    from oracle import transformer_layer as T
    g = np.random.default_rng(12)
    S, hq, hkv, d = 7, 2, 2, 4
    H = hq * d
    p = {"w_qkv": g.normal(size=(H, 3 * H)), "w_o": g.normal(size=(H, H)), "w_1": g.normal(size=(H, 4 * H)),
         "w_2": g.normal(size=(4 * H, H)), "g1": g.normal(size=H), "b1": g.normal(size=H), "g2": g.normal(size=H),
         "b2": g.normal(size=H)}
    x, dy = g.normal(size=(S, H)), g.normal(size=(S, H))
    a = T.layer(x, dy, p, hq, hkv, d)
    one = np.ones((S, H))
    b = O.layer_with_ends(x, dy, p, hq, hkv, d, dict(norm="none", gate=False, alpha=1.0, scale=1.0), one, one)
    for k in a:
        np.testing.assert_allclose(a[k], b[k], rtol=1e-12, atol=1e-12 * np.abs(a[k]).max())


# ------------------------------------------------------------------ refusals
A = 4096  # any aligned non-null address: nothing is launched on a refusal


def refused(status, fn, *args, **kw):
    with pytest.raises(L.SppoError) as e:
        fn(*args, **kw)
    assert e.value.status == status
    assert L.sppo_last_error(None)


def test_struct_layouts_match_c():
    assert ctypes.sizeof(L.sppo_drop) == 40 and L.sppo_drop.row0.offset == 32
    assert ctypes.sizeof(L.sppo_block_norm) == 72 and L.sppo_block_norm.post_gamma.offset == 32
    assert ctypes.sizeof(L.sppo_block_norm_stats) == 32 and ctypes.sizeof(L.sppo_block_norm_grads) == 40


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), BAD), (dict(rows=-1), BAD), (dict(cols=12), BAD), (dict(cols=0), BAD), (dict(dtype=5), BAD),
    (dict(x=None), BAD), (dict(x=A + 8), BAD), (dict(y=None), BAD), (dict(ldx=56), BAD), (dict(ldx=68), BAD),
    (dict(ldy=60), BAD), (dict(res=A + 4), BAD), (dict(res=A, ldres=8), BAD), (dict(p=-0.1), BAD), (dict(p=1.0), BAD),
    (dict(p=float("nan")), BAD), (dict(p=0.999999), BAD), (dict(row0=-1), BAD), (dict(offset_dev=A + 4), BAD),
    (dict(nodrop=True), BAD), (dict(row0=2 ** 62), UNSUP), (dict(row0=2 ** 63 - 1), UNSUP),
])
def test_dropout_refuses(change, status):
    a = dict(rows=4, cols=64, x=A, ldx=64, y=A, ldy=64, res=None, ldres=64, dtype="bf16", p=0.1, row0=0,
             offset_dev=None, nodrop=False)
    a.update(change)
    d = None if a["nodrop"] else L.drop_spec(a["p"], 1, 2, a["row0"], a["offset_dev"])
    refused(status, L.sppo_dropout, a["rows"], a["cols"], a["x"], a["ldx"], d, a["y"], a["ldy"], a["res"], a["ldres"],
            a["dtype"], stream=0)


FULL = dict(post="layer", pre="layer", gate_kind="channel", post_gamma=A, post_beta=A, gate=A, pre_gamma=A, pre_beta=A)


@pytest.mark.parametrize("change,status", [
    (dict(H=12), BAD), (dict(H=8200), BAD), (dict(H=0), BAD), (dict(dtype=9), BAD), (dict(post=3), BAD),
    (dict(pre=-1), BAD), (dict(gate_kind=7), BAD), (dict(eps=0.0), BAD), (dict(eps=float("inf")), BAD), (dict(eps=1e-40), BAD),
    (dict(residual_scale=float("nan")), BAD), (dict(branch_scale=float("inf")), BAD), (dict(branch_scale=-1e34), BAD), (dict(post_gamma=None), BAD),
    (dict(pre_gamma=None), BAD), (dict(gate=None), BAD), (dict(pre_beta=A + 2), BAD),
])
def test_block_norm_refuses_a_bad_description(change, status):
    kw = dict(FULL, H=64, dtype="bf16")
    kw.update(change)
    bn = L.block_norm(**kw)
    st = L.block_norm_stats(A, A, A, A)
    refused(status, L.sppo_block_norm_fwd, bn, 4, None, A, 64, A, 64, A, 64, 2 * A, 64, st, stream=0)
    assert L.sppo_block_norm_bwd_workspace(bn, 4) == 0
    refused(status, L.sppo_block_norm_bwd, bn, 4, None, A, 64, A, 64, st, A, 64, A, 64, A, 64, 2 * A, 64, None, A,
            1 << 30, stream=0)


def test_block_norm_refuses_bad_calls():
    bn = L.block_norm(64, **FULL)
    st = L.block_norm_stats(A, A, A, A)
    fwd = lambda rows=4, drop=None, x=A, ldx=64, b=A, h=A, z=2 * A, stats=st, bn=bn: L.sppo_block_norm_fwd(
        bn, rows, drop, x, ldx, b, 64, h, 64, z, 64, stats, stream=0)
    for kw in (dict(rows=0), dict(x=None), dict(ldx=60), dict(ldx=68), dict(b=A + 8), dict(h=None), dict(z=None),
               dict(z=A), dict(stats=None), dict(stats=L.block_norm_stats(None, A, A, A)),
               dict(stats=L.block_norm_stats(A, A, A, None)), dict(drop=L.drop_spec(1.5, 0))):
        refused(BAD, fwd, **kw)
    refused(UNSUP, fwd, rows=1 << 22)
    gr = L.block_norm_grads(A, A, A, A, A)
    ws = L.sppo_block_norm_bwd_workspace(bn, 4)
    assert ws > 0
    bwd = lambda b=A, h=A, stats=st, dz=A, dh=A, dx=A, db=2 * A, grads=gr, w=A, nb=ws, acc=0, bn=bn: \
        L.sppo_block_norm_bwd(bn, 4, None, b, 64, h, 64, stats, dz, 64, dh, 64, dx, 64, db, 64, grads, w, nb, acc,
                              stream=0)
    for kw in (dict(b=None), dict(h=None), dict(dz=None), dict(dx=None), dict(db=None), dict(db=A), dict(dh=A + 2),
               dict(w=None), dict(w=A + 4), dict(nb=ws - 1), dict(acc=2), dict(stats=None),
               dict(grads=L.block_norm_grads(A + 1))):
        refused(BAD, bwd, **kw)
    # without a norm in front of the next block the gradient has to come through dh
    plain = L.block_norm(64, post="layer", post_gamma=A)
    refused(BAD, bwd, bn=plain, dh=None)


def test_block_norm_workspace_grows_with_rows():
    for H in (64, 1024, 4096):
        bn = L.block_norm(H, **FULL)
        sizes = [L.sppo_block_norm_bwd_workspace(bn, r) for r in list(range(1, 3000)) + [8192, 65536, 1 << 21]]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), BAD), (dict(V=0), BAD), (dict(H=20), BAD), (dict(H=0), BAD), (dict(ids=None), BAD),
    (dict(ids=A + 4), BAD), (dict(dtype=4), BAD), (dict(id_type=2), BAD), (dict(scale=float("nan")), BAD), (dict(scale=1e34), BAD),
    (dict(act=None), BAD), (dict(act=A + 8), BAD), (dict(ld=56), BAD), (dict(table=None), BAD), (dict(table=A + 4), BAD),
    (dict(ldt=60), BAD), (dict(p=1.0), BAD), (dict(rows=(1 << 28) + 1), UNSUP), (dict(V=1 << 31), UNSUP),
    (dict(rows=1 << 28, H=1032, ld=1032, ldt=1032), UNSUP),
    (dict(H=(1 << 20) + 8, ld=1 << 21, ldt=1 << 21), UNSUP),
])
def test_embedding_refuses(change, status):
    a = dict(rows=4, H=64, V=100, ids=A, table=A, ldt=64, scale=1.0, act=A, ld=64, dtype="bf16", id_type="i64", p=0.1)
    a.update(change)
    d = L.drop_spec(a["p"], 1)
    refused(status, L.sppo_embedding_fwd, a["rows"], a["H"], a["V"], a["ids"], a["table"], a["ldt"], a["scale"], d,
            a["act"], a["ld"], a["dtype"], a["id_type"], stream=0)
    refused(status, L.sppo_embedding_bwd, a["rows"], a["H"], a["V"], a["ids"], a["act"], a["ld"], a["scale"], d,
            a["table"], a["ldt"], A, 1 << 40, 0, a["dtype"], a["id_type"], stream=0)


def test_embedding_refuses_bad_workspaces():
    ws = L.sppo_embedding_bwd_workspace(4, 64)
    assert ws > 0 and L.sppo_embedding_bwd_workspace(0, 64) == 0 and L.sppo_embedding_bwd_workspace(4, 12) == 0
    call = lambda w, n, acc=0: L.sppo_embedding_bwd(4, 64, 100, A, A, 64, 1.0, None, A, 64, w, n, acc, stream=0)
    refused(BAD, call, None, ws)
    refused(BAD, call, A + 8, ws)
    refused(BAD, call, A, ws - 1)
    refused(BAD, call, A, ws, 2)
    sizes = [L.sppo_embedding_bwd_workspace(r, 256) for r in range(1, 5000)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("change", [
    dict(dropout=0.999999), dict(dropout=-0.1), dict(dropout=float("nan")), dict(residual_scale=float("inf")),
    dict(residual_scale=float("nan")), dict(branch_scale=float("nan")), dict(branch_scale=-(2.0 ** 112)),
    dict(branch_scale=1e39), dict(residual_scale=1e39),
])
def test_block_ends_refuse_what_the_calls_would(change):
    """What sppo_drop and sppo_block_norm refuse is refused before a walk begins."""
    from paper_2503_10377_amd.chunked_layer import BlockEnds
    with pytest.raises(ValueError):
        BlockEnds(**change)


def test_block_ends_take_what_the_calls_take():
    from paper_2503_10377_amd.chunked_layer import BlockEnds
    for kw in (dict(dropout=65535 / 65536), dict(branch_scale=2.0 ** 111), dict(residual_scale=-3e38), dict()):
        BlockEnds(**kw)
    assert [L.drop_threshold(p) for p in (0.0, 0.5, 65535 / 65536)] == [O.threshold(p) for p in (0.0, 0.5, 65535 / 65536)]


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), 2.0 ** 112])
def test_layer_refuses_an_embedding_scale_that_the_call_would(scale):
    from paper_2503_10377_amd.chunked_layer import ChunkedLayer
    with pytest.raises(ValueError):
        ChunkedLayer(256, 1, 2, 2, 128, vocab=10, embed_scale=scale, device="cpu")
