"""Pins of the step operators' oracle, their host functions, and what the calls
refuse (on the CPU: nothing is enqueued)."""
import ctypes
import math

import numpy as np
import pytest

from oracle import step_ops as O
from paper_2503_10377_amd import sppo as L

BAD, UNS = L.SPPO_ERR_INVALID_ARG, L.SPPO_ERR_UNSUPPORTED


# ------------------------------------------------------------------- the oracle
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_keeps_lengths_and_differences(layout):
    r = np.random.RandomState(0)
    f, _ = O.rope_freqs(16)
    x, y = r.randn(1, 2, 24), r.randn(1, 2, 24)
    at = lambda v, p: O.rotary(v, [p], f, 16, layout)  # noqa: E731
    assert np.allclose((at(x, 77) ** 2).sum(), (x ** 2).sum())
    assert np.allclose(at(x, 77)[..., 16:], x[..., 16:])
    assert np.allclose(O.rotary(at(x, 77), [77], f, 16, layout, inverse=True), x)
    dots = [(at(x, 5 + k) * at(y, 17 + k)).sum() for k in (0, 3, 1000)]
    assert np.allclose(dots, dots[0])
    # The pair of the fastest frequency turns by one radian a position.
    a, b = (0, 8) if layout == "half" else (0, 1)
    e = np.zeros((1, 1, 16))
    e[..., a] = 1.0
    out = O.rotary(e, [1], f, 16, layout)
    assert np.allclose([out[0, 0, a], out[0, 0, b]], [math.cos(1), math.sin(1)])


def test_cross_entropy_against_a_loop_and_differences():
    r = np.random.RandomState(1)
    x, t = r.randn(3, 7), np.array([2, -1, 6])
    e, z = 0.2, 0.01
    loss, lse, dx = O.cross_entropy(x, t, e, z, 1.0)
    for i in (0, 2):
        want = -math.log(sum(math.exp(v) for v in x[i])) * -1
        nll = [want - v for v in x[i]]
        assert np.isclose(loss[i], (1 - e) * nll[t[i]] + e / 7 * sum(nll) + z * want ** 2)
        for c in range(7):
            h = np.zeros_like(x)
            h[i, c] = 1e-5
            d = (O.cross_entropy(x + h, t, e, z)[0][i] - O.cross_entropy(x - h, t, e, z)[0][i]) / 2e-5
            assert np.isclose(dx[i, c], d, atol=1e-8)
    assert loss[1] == lse[1] == 0 and not dx[1].any()


def test_adamw_against_a_loop():
    p, g, m, v = 0.5, [0.3, -0.2, 0.1], 0.0, 0.0
    P, M, V = np.array([p]), np.zeros(1), np.zeros(1)
    for t, gt in enumerate(g, 1):
        m, v = 0.9 * m + 0.1 * gt, 0.99 * v + 0.01 * gt ** 2
        p -= 0.01 * (m / (1 - 0.9 ** t) / (math.sqrt(v / (1 - 0.99 ** t)) + 1e-8) + 0.1 * p)
        P, M, V = O.adamw(P, np.array([gt]), M, V, t, 0.01, 0.9, 0.99, 1e-8, 0.1)
    assert np.isclose(P[0], p) and np.isclose(M[0], m) and np.isclose(V[0], v)


def test_eight_bit_format_and_rounding():
    assert O.E4M3[0] == 0 and O.E4M3[1] == 2.0 ** -9 and O.E4M3[8] == 2.0 ** -6 and O.E4M3[126] == 448
    assert (np.diff(O.E4M3) > 0).all()
    x = np.zeros(64)
    x[:4] = [448.0, -448.0, 1.0, 0.0]
    x[32] = 449.0
    assert O.block_bytes(x).tolist() == [127, 128]
    assert O.block_bytes(np.zeros(5)).tolist() == [1]
    # The mean over all draws is the value to 2^-16 of a step.
    u = np.arange(65536)
    for v, step in ((1.06, 0.125), (-3.3, 0.25), (0.003, 2.0 ** -9), (300.0, 32.0)):
        codes, _ = O.round8(np.full(65536, v), np.full(2048, 127, np.uint8), u, False)
        mean = O.value8(codes, np.full(2048, 127, np.uint8)).mean()
        assert abs(mean - v) <= step / 65536, v
    codes, _ = O.round8(np.full(32, 1e-6), np.array([127], np.uint8), np.zeros(32), True)
    assert (codes == 1).all()


def test_layer_step_gradients_by_differences():
    r = np.random.RandomState(3)
    hq, hkv, d, S, C = 2, 1, 8, 5, 11
    H = hq * d
    shapes = dict(w_qkv=(H, (hq + 2 * hkv) * d), w_o=(H, H), w_1=(H, 4 * H), w_2=(4 * H, H), w_out=(H, C), g1=H, b1=H,
                  g2=H, b2=H, gf=H, bf=H)
    p = {k: r.randn(*(v if isinstance(v, tuple) else (v,))) * (0.3 if k[0] == "w" else 1.0) for k, v in shapes.items()}
    x, t = r.randn(S, H), np.array([3, -1, 10, 0, 3])
    rope = dict(rot=8, layout="interleaved", freqs=O.rope_freqs(8)[0], amp=1.1, position0=7)
    run = lambda x, p: O.layer_step(x, p, hq, hkv, d, rope, t, 0.1, 0.01, 0.2)  # noqa: E731
    out = run(x, p)
    f = lambda x, p: 0.2 * run(x, p)["loss"].sum()  # noqa: E731
    for name in ["x", *p]:
        v = x if name == "x" else p[name]
        for i in r.choice(v.size, 4, replace=False):
            h = np.zeros(v.size)
            h[i] = 1e-5
            h = h.reshape(v.shape)
            d2 = (f(x + h, p) - f(x - h, p)) if name == "x" else (f(x, {**p, name: v + h}) - f(x, {**p, name: v - h}))
            assert np.isclose(out["d" + name].ravel()[i], d2 / 2e-5, rtol=1e-5, atol=1e-8), (name, i)


# --------------------------------------------------------------- host functions
@pytest.mark.parametrize("rot", [8, 24, 128, 1024])
@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0),
                                dict(scaling="ntk", factor=8.0),
                                dict(scaling="yarn", factor=16.0, original_len=4096.0),
                                dict(scaling="yarn", factor=1.0, original_len=100.0, beta_fast=8.0, beta_slow=2.0)])
def test_rotary_freqs(rot, kw):
    got, amp = L.sppo_rotary_freqs(rot, **kw)
    o = dict(kw)
    o["kind"] = o.pop("scaling", "none")
    f, want_amp = O.rope_freqs(rot, **o)
    turns = (f / (2 * np.longdouble("3.14159265358979323846264338327950288"))).tolist()
    assert abs(amp - want_amp) <= 2.0 ** -24 * want_amp
    for a, b in zip(got, turns):
        assert abs(np.longdouble(a) - np.longdouble(b) * np.longdouble(2.0 ** 64)) <= 2 ** 12  # the oracle's powers


def test_rotary_freqs_given():
    given = [0.0, 1.0, -1.0, 2 * math.pi, 0.25]
    got, amp = L.sppo_rotary_freqs(10 - 2, scaling="given", inv_freq=given[:4])
    assert amp == 1.0 and got[0] == 0
    assert got[1] + got[2] == 2 ** 64
    assert abs(got[1] / 2.0 ** 64 - 1 / (2 * math.pi)) < 1e-16
    assert min(got[3], 2 ** 64 - got[3]) < 2 ** 13  # a double's 2 pi is off by up to 2^-51
    with pytest.raises(ValueError):
        L.sppo_rotary_freqs(8, scaling="given", inv_freq=given)


def test_rotary_freqs_drop_nothing_that_is_given():
    """inv_freq alone is the table; settings that nothing would read are refused,
    by the layer's description too."""
    from paper_2503_10377_amd.chunked_layer import Rotary

    given = [0.5, 0.25, -0.125, 3.0]
    want = L.sppo_rotary_freqs(8, scaling="given", inv_freq=given)
    assert want != L.sppo_rotary_freqs(8)
    assert L.sppo_rotary_freqs(8, inv_freq=given) == want
    rot, table, amp = Rotary(inv_freq=given).table(8, "cpu")
    assert table.numpy().view(np.uint64).tolist() == want[0] and amp == 1.0
    for kw in (dict(scaling="none", inv_freq=given), dict(scaling="yarn", factor=2.0, original_len=64, inv_freq=given),
               dict(inv_freq=given, factor=2.0), dict(inv_freq=given, base=500000.0), dict(factor=8.0),
               dict(original_len=4096.0), dict(beta_fast=16.0), dict(beta_slow=2.0)):
        with pytest.raises(ValueError):
            L.sppo_rotary_freqs(8, **kw)
        with pytest.raises(ValueError):
            Rotary(**kw).table(8, "cpu")
    # A scaling that is named says which settings count.
    assert L.sppo_rotary_freqs(8, 10000.0, "none", factor=8.0, original_len=4096.0) == L.sppo_rotary_freqs(8)


@pytest.mark.parametrize("kw", [
    dict(rot=0), dict(rot=12), dict(rot=1032), dict(rot=-8), dict(base=1.0), dict(base=float("inf")),
    dict(base=float("nan")), dict(scaling=9), dict(scaling="linear", factor=0.5),
    dict(scaling="ntk", factor=float("nan")), dict(scaling="yarn", factor=2.0),
    dict(scaling="yarn", factor=2.0, original_len=10.0, beta_fast=1.0), dict(scaling="given"),
    dict(scaling="given", inv_freq=[1.0, float("inf"), 0.0, 0.0]),
])
def test_rotary_freqs_refuses(kw):
    kw = {"rot": 8, **kw}
    with pytest.raises(L.SppoError) as e:
        L.sppo_rotary_freqs(**kw)
    assert e.value.status == BAD and L.sppo_last_error(None)


def tensors(sizes, state="f32", param="bf16", grad="f32"):
    """opt_tensor()s at made-up addresses."""
    at, out = 1 << 20, []

    def take(n):
        nonlocal at
        a, at = at, (at + n + 255) // 256 * 256
        return a

    for n in sizes:
        kw = dict(grad=take(4 * n), grad_dtype=grad, param=take(4 * n), param_dtype=param,
                  master=take(4 * n) if param == "bf16" else None, m=take(4 * n), v=take(4 * n))
        if state == "e4m3":
            kw.update(m_scale=take(n), v_scale=take(n))
        out.append(L.opt_tensor(n, **kw))
    return out


def make(ts, state="f32", short=0):
    nbytes = max(16, L.sppo_opt_list_bytes(ts) - short)
    host = (ctypes.c_uint64 * (nbytes // 8 + 2))(*[0xABABABABABABABAB] * (nbytes // 8 + 2))
    out = L.sppo_opt_list_make(ts, state, ctypes.addressof(host), nbytes)
    assert bytes(host)[max(nbytes, 16):] == b"\xab" * (len(bytes(host)) - max(nbytes, 16)), "written past the table"
    return out, host


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_opt_list(state):
    ts = tensors([1, 0, 4096, 4097, 70000], state)
    got, host = make(ts, state)
    assert (got.tiles, got.n_tensors, got.state) == (1 + 0 + 2 + 3 + 35, 5, L.OPT_STATES[state])
    tiles = np.frombuffer(host, dtype=np.uint32)[5 * 96 // 4:][:2 * got.tiles].reshape(-1, 2)
    assert tiles[:5].tolist() == [[0, 0], [2, 0], [2, 1], [3, 0], [3, 1]] and tiles[-1].tolist() == [4, 34]
    block0 = [int.from_bytes(bytes(host)[96 * i + 64:96 * i + 72], "little") for i in range(5)]
    assert block0 == [0, 1, 1, 129, 129 + 129]


def change(ts, i, **kw):
    for k, v in kw.items():
        setattr(ts[i], k, v)
    return ts


@pytest.mark.parametrize("build,status", [
    (lambda: change(tensors([8]), 0, n=-1), BAD),
    (lambda: change(tensors([8]), 0, grad=None), BAD),
    (lambda: change(tensors([8]), 0, grad=(1 << 20) + 2), BAD),
    (lambda: change(tensors([8]), 0, grad_dtype=5), BAD),
    (lambda: change(tensors([8]), 0, param_dtype=5), BAD),
    (lambda: change(tensors([8]), 0, param=None), BAD),
    (lambda: change(tensors([8]), 0, m=None), BAD),
    (lambda: change(tensors([8]), 0, v=6), BAD),
    (lambda: change(tensors([8]), 0, master=None), BAD),
    (lambda: change(tensors([8], param="f32"), 0, master=1 << 30), BAD),
    (lambda: change(tensors([8]), 0, lr_scale=float("inf")), BAD),
    (lambda: change(tensors([8]), 0, weight_decay=float("nan")), BAD),
    (lambda: tensors([8]) * 2, BAD),                                     # listed twice
    (lambda: (lambda t: change(t, 0, m=t[1].param))(tensors([8, 8])), BAD),
    (lambda: (lambda t: change(t, 0, v=t[0].m + 16))(tensors([8])), BAD),  # v inside m
    (lambda: (lambda t: change(t, 0, grad=t[1].master))(tensors([8, 8])), BAD),
    (lambda: change(tensors([8, 8]), 1, n=2 ** 36), UNS),
])
def test_opt_list_refuses(build, status):
    with pytest.raises(L.SppoError) as e:
        make(build())
    assert e.value.status == status


def test_opt_list_allows():
    """Shared gradients; neighbours without a gap; the last two of 8-bit states'
    own demands refused."""
    t = tensors([8, 8])
    make(change(t, 1, grad=t[0].grad))
    make(change(t, 1, m=t[0].m + 32))
    t = tensors([8], "none")
    make(change(t, 0, param=None, m=None, v=None, master=None), "none")
    for k, v in (("m", (1 << 20) + 8), ("m_scale", None)):
        with pytest.raises(L.SppoError):
            make(change(tensors([8], "e4m3"), 0, **{k: v}), "e4m3")
    with pytest.raises(L.SppoError):
        make(tensors([8]), short=8)
    with pytest.raises(L.SppoError):
        make([])
    assert L.sppo_opt_list_bytes([]) == 0


# -------------------------------------------------------------------- refusals
P = 1 << 20  # an address that no call gets to use


def rot_call(spec=None, t=None, rows=4, inverse=0, n=1, **over):
    s = dict(rot=16, freqs=P, layout="half", amp=1.0, positions=None)
    s.update(spec or {})
    d = dict(heads=2, head_dim=32, x=P, ldx=64, hsx=32, y=2 * P, ldy=64, hsy=32, dtype="bf16")
    d.update(t or {})
    L.sppo_rotary_apply(L.rotary(**s), rows, L.rotary_tensors([L.rotary_tensor(**d)] * n), inverse, stream=0)


@pytest.mark.parametrize("kw,status", [
    (dict(spec=dict(rot=12)), BAD), (dict(spec=dict(rot=0)), BAD), (dict(spec=dict(rot=40)), BAD),
    (dict(spec=dict(layout=2)), BAD), (dict(spec=dict(freqs=None)), BAD), (dict(spec=dict(freqs=P + 4)), BAD),
    (dict(spec=dict(amp=float("nan"))), BAD), (dict(spec=dict(positions=P + 4)), BAD),
    (dict(spec=dict(id_type=4)), BAD), (dict(rows=-1), BAD), (dict(inverse=2), BAD), (dict(n=5), BAD),
    (dict(n=2), BAD),                            # the same tensor twice
    (dict(t=dict(dtype=3)), BAD), (dict(t=dict(heads=0)), BAD), (dict(t=dict(head_dim=20)), BAD),
    (dict(t=dict(head_dim=1032, hsx=1032, hsy=1032, ldx=4096, ldy=4096)), UNS),
    (dict(t=dict(heads=65536, ldx=2 ** 30, ldy=2 ** 30)), UNS),
    (dict(t=dict(x=None)), BAD), (dict(t=dict(y=P + 8)), BAD), (dict(t=dict(ldx=60)), BAD),
    (dict(t=dict(ldx=56)), BAD),                 # rows over one another
    (dict(t=dict(hsy=24)), BAD),                 # heads over one another
    (dict(t=dict(ldx=2 ** 60)), BAD),
    (dict(t=dict(y=P, ldy=72)), BAD),            # over x with other strides
    (dict(t=dict(ldx=32, hsx=96)), BAD),         # head-major, but three rows' space for four
])
def test_rotary_refuses(kw, status):
    with pytest.raises(L.SppoError) as e:
        rot_call(**kw)
    assert e.value.status == status and L.sppo_last_error(None)


def test_calls_on_no_rows_do_nothing():
    rot_call(rows=0)
    ce = L.cross_entropy(10)
    L.sppo_cross_entropy(ce, 0, P, 16, P, P, P, P, 16, stream=0)
    L.sppo_cross_entropy_bwd(ce, 0, P, 16, P, P, None, P, 16, stream=0)
    empty, host = make(tensors([0, 0]))
    empty.table = P
    L.sppo_adamw_step(empty, L.adamw(1e-3), stream=0)


@pytest.mark.parametrize("spec,call,status", [
    (dict(V=0), {}, BAD), (dict(V=2 ** 31), {}, UNS), (dict(dtype=4), {}, BAD), (dict(id_type=4), {}, BAD),
    (dict(label_smoothing=-0.1), {}, BAD), (dict(label_smoothing=1.1), {}, BAD),
    (dict(label_smoothing=float("nan")), {}, BAD), (dict(z_loss=-1.0), {}, BAD), (dict(z_loss=float("inf")), {}, BAD),
    (dict(scale=float("nan")), {}, BAD), (dict(scale_dev=P + 2), {}, BAD),
    ({}, dict(rows=-1), BAD), ({}, dict(rows=2 ** 31), UNS), ({}, dict(logits=None), BAD),
    ({}, dict(logits=P + 8), BAD),
    ({}, dict(ld=12), BAD), ({}, dict(ld=8), BAD), ({}, dict(ld=2 ** 62), BAD), ({}, dict(targets=None), BAD),
    ({}, dict(targets=P + 4), BAD), ({}, dict(loss=None), BAD), ({}, dict(loss=P + 2), BAD), ({}, dict(lse=P + 1), BAD),
    ({}, dict(dlogits=P + 8), BAD), ({}, dict(lddl=8), BAD), ({}, dict(dlogits=P, lddl=24), BAD),
])
def test_cross_entropy_refuses(spec, call, status):
    ce = L.cross_entropy(**{"V": 10, **spec})
    c = dict(rows=4, logits=P, ld=16, targets=2 * P, loss=3 * P, lse=4 * P, dlogits=5 * P, lddl=16)
    c.update(call)
    with pytest.raises(L.SppoError) as e:
        L.sppo_cross_entropy(ce, *c.values(), stream=0)
    assert e.value.status == status and L.sppo_last_error(None)
    if "loss" in call or call.get("lse") == P + 1:
        return
    del c["loss"]
    c = {k: c.get(k) for k in ("rows", "logits", "ld", "targets", "lse", "dloss", "dlogits", "lddl")}
    with pytest.raises(L.SppoError) as e:
        L.sppo_cross_entropy_bwd(ce, *c.values(), stream=0)
    assert e.value.status == status


def test_cross_entropy_bwd_refuses():
    for lse, dloss, dl in ((None, None, P), (P + 2, None, P), (P, P + 2, P), (P, None, None)):
        with pytest.raises(L.SppoError) as e:
            L.sppo_cross_entropy_bwd(L.cross_entropy(10), 4, 2 * P, 16, 3 * P, lse, dloss, dl, 16, stream=0)
        assert e.value.status == BAD


def test_update_refuses():
    lst, host = make(tensors([100]))
    with pytest.raises(L.SppoError):        # no table on the device yet
        L.sppo_adamw_step(lst, L.adamw(1e-3), stream=0)
    lst.table = P
    for kw in (dict(lr=float("nan")), dict(lr=1e300), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0),
               dict(eps=0.0), dict(eps=1e-40), dict(eps=float("inf")), dict(step=0), dict(step_dev=P + 4), dict(norm=P + 2),
               dict(lr_dev=P + 2)):
        with pytest.raises(L.SppoError) as e:
            L.sppo_adamw_step(lst, L.adamw(**{"lr": 1e-3, **kw}), stream=0)
        assert e.value.status == BAD, kw
    grads, host2 = make(tensors([100]), "none")
    grads.table = P
    with pytest.raises(L.SppoError):
        L.sppo_adamw_step(grads, L.adamw(1e-3), stream=0)
    need = L.sppo_grad_norm_workspace(grads)
    assert need > 0 and L.sppo_grad_norm_workspace(None) == 0
    ok = dict(max_norm=1.0, out=P, workspace=P, workspace_bytes=need, steps=None)
    for kw in (dict(max_norm=0.0), dict(max_norm=float("nan")), dict(out=None), dict(out=P + 2), dict(workspace=None),
               dict(workspace=P + 8), dict(workspace_bytes=need - 1), dict(steps=P + 4)):
        with pytest.raises(L.SppoError) as e:
            L.sppo_grad_norm(grads, **{**ok, **kw}, stream=0)
        assert e.value.status == BAD, kw


def test_struct_layouts_match_c():
    assert ctypes.sizeof(L.sppo_rotary) == 40 and ctypes.sizeof(L.sppo_rotary_tensor) == 64
    assert ctypes.sizeof(L.sppo_rope) == 56 and ctypes.sizeof(L.sppo_ce) == 40
    assert ctypes.sizeof(L.sppo_opt_tensor) == 80 and ctypes.sizeof(L.sppo_opt_list) == 24
    assert ctypes.sizeof(L.sppo_adamw) == 72


def test_layer_refuses_before_the_device():
    """What the layer's options say for themselves."""
    from paper_2503_10377_amd.chunked_layer import Loss, Rotary
    from paper_2503_10377_amd.optimizer import AdamW
    import torch

    for kw in (dict(layout="spiral"), dict(position0=-1), dict(position0=2 ** 62)):
        with pytest.raises(ValueError):
            Rotary(**kw)
    with pytest.raises(ValueError):
        Rotary(rot=128).table(64, "cpu")
    with pytest.raises(L.SppoError):
        Rotary(rot=20).table(64, "cpu")
    rot, table, amp = Rotary(base=500000.0).table(64, "cpu")
    assert rot == 64 and table.shape == (32,) and amp == 1.0
    for a in ((0,), (100,), (2 ** 31,), (256, -0.1), (256, 0.0, -1.0), (256, 0.0, float("nan")), (256, 0.0, 1e39)):
        with pytest.raises(ValueError):
            Loss(*a)
    w = torch.zeros(4)
    for params, grads, kw in (({}, {}, {}), ({"a": w}, {"b": w}, {}), ({"a": w}, {"a": w}, {}),
                              ({"a": w}, {"a": w}, dict(state="f16")), ({"a": w}, {"a": w}, dict(max_norm=0.0)),
                              ({"a": w}, {"a": w}, dict(betas=(0.9, 1.0))), ({"a": w}, {"a": w}, dict(eps=0.0))):
        with pytest.raises(ValueError):
            AdamW(params, grads, 1e-3, **kw)


def test_optimizer_needs_two_betas():
    from paper_2503_10377_amd.optimizer import AdamW
    import torch

    w = torch.zeros(4)
    for betas in ((), (0.9,), (0.9, 0.95, 0.99)):
        with pytest.raises(ValueError, match="betas"):
            AdamW({"a": w}, {"a": w}, 1e-3, betas=betas)


def test_optimizer_refuses_an_eps_that_the_update_refuses():
    """eps as the update's call takes it: a normal fp32 number."""
    from paper_2503_10377_amd.optimizer import AdamW
    import torch

    w = torch.zeros(4)
    for eps in (1e-46, 1e-40, 2.0 ** -126 * (1 - 2.0 ** -20), 1e39, float("inf"), float("nan"), 0.0, -1e-8):
        with pytest.raises(ValueError, match="eps"):
            AdamW({"a": w}, {"a": w}, 1e-3, eps=eps)
    for eps in (2.0 ** -126, 1e-8, 1.0):  # refused for their tensors, which are in host memory
        with pytest.raises(ValueError, match="device"):
            AdamW({"a": w}, {"a": w}, 1e-3, eps=eps)


@pytest.mark.parametrize("heads,classes", [(64, 2 ** 18), (32, 2 ** 19), (2, 2 ** 22), (2, 2 ** 30)])
def test_layer_refuses_classes_that_its_products_refuse(heads, classes):
    """The gradient of [H, classes] weights counts its elements in 31 bits, and a
    product over the classes takes fewer than 2^22: refused with the layer, not in
    the last chunk of its first step.  The products' calls refuse the same sizes."""
    from paper_2503_10377_amd.chunked_layer import ChunkedLayer, Loss

    H = 128 * heads
    with pytest.raises(ValueError, match="classes"):
        ChunkedLayer(512, 4, heads, heads, 128, device="cpu", loss=Loss(classes))

    call = ("tn", H, classes, 128, P, H, P, classes, P, classes)
    if H * classes < 2 ** 31:
        call = ("nt", 128, H, classes, P, classes, P, classes, P, H)
    with pytest.raises(L.SppoError) as e:
        L.sppo_gemm_bf16(*call, stream=0)
    assert e.value.status == UNS


def test_cross_entropy_workspace_is_asked_for_where_it_is_used():
    """Few long rows and rows past 131072 bf16 (65536 fp32) logits need it; the
    size never shrinks with more rows, so one for the largest call serves all."""
    for V, dtype, first in ((32768, "bf16", None), (32769, "bf16", 1), (131072, "bf16", 1), (65536, "f32", 1),
                            (131073, "bf16", 1), (65537, "f32", 1)):
        ce = L.cross_entropy(V, dtype)
        sizes = [L.sppo_cross_entropy_workspace(ce, r) for r in (0, 1, 2, 126, 127, 128, 129, 5000)]
        assert sizes == sorted(sizes) and sizes[0] == 0 and (sizes[1] > 0) == (first == 1)
    c = dict(logits=P, ld=131080, targets=2 * P, loss=3 * P, lse=None, dlogits=None, lddl=0)
    for V, rows in ((40001, 1), (40001, 127), (131073, 128), (131073, 5000)):
        ce = L.cross_entropy(V)
        need = L.sppo_cross_entropy_workspace(ce, rows)
        for ws, n in ((None, 0), (None, need), (P, need - 1), (P + 8, need)):
            with pytest.raises(L.SppoError) as e:
                L.sppo_cross_entropy(ce, rows, *c.values(), ws, n, stream=0)
            assert e.value.status == BAD


def test_rotary_amplitude_of_given_frequencies():
    """Given frequencies have the amplitude that is given with them."""
    from paper_2503_10377_amd.chunked_layer import Rotary

    given = [0.5, 0.25, -0.125, 3.0]
    assert Rotary(inv_freq=given, amp=1.25).table(8, "cpu")[2] == 1.25
    assert Rotary(scaling="yarn", factor=4.0, original_len=64, amp=1.0).table(8, "cpu")[2] == 1.0
    for amp in (float("inf"), float("nan"), 1e39):
        with pytest.raises(ValueError):
            Rotary(inv_freq=given, amp=amp)
