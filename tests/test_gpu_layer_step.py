"""A training step of the chunked layer: rotary positions in its attention, the
loss of its output chunk by chunk, and the update of its parameters, against
the fp64 oracle; results do not depend on what is offloaded.

Gates as in test_gpu_layer.py (bf16 activations at every step): per tensor,
relative Frobenius error <= 1.2e-2 and max |err| <= 1.5e-2 of max |ref|.  The
rotations round q and k, dq and the packed dk once more each, the logits and
their gradient round like the layer's other activations.  A rotation at another
position or in the wrong sense, a missing factor or a target off by one moves
its outputs by O(1).
"""
import sys

import numpy as np
import pytest
import torch

from oracle import step_ops as O
from oracle import train_ops as T
from paper_2503_10377_amd import chunked_layer as C
from paper_2503_10377_amd import sppo as L
from paper_2503_10377_amd.chunked_layer import BlockEnds, ChunkedLayer, Loss, Rotary
from paper_2503_10377_amd.inputs import make_layer_inputs
from paper_2503_10377_amd.optimizer import AdamW
from parity import to_np

pytestmark = pytest.mark.gpu
REL, MAXREL = 1.2e-2, 1.5e-2
INF = float("inf")


def announce(msg):
    print(f"\n[case] {msg}", file=sys.stderr, flush=True)


def setup(S, Hq, Hkv, D, classes, vocab, seed, ends=None, ids=torch.int64):
    inp, p = make_layer_inputs(S, Hq, Hkv, D, seed, device="cpu")
    H = Hq * D
    g = torch.Generator().manual_seed(2000 + seed)
    for n in (1, 2):
        for k, name in ends.params(n).items() if ends is not None else ():
            r = torch.randn(H, generator=g)
            p[name] = 0.1 * r if k == "post_beta" else 1.0 + 0.1 * r
    if classes is not None:
        p["w_out"] = (torch.randn(H, classes, generator=g) * H ** -0.5).to(torch.bfloat16)
        p["gf"], p["bf"] = 1.0 + 0.1 * torch.randn(H, generator=g), 0.1 * torch.randn(H, generator=g)
        t = torch.randint(0, classes, (S,), generator=g)
        t[::9] = -1
        inp = {"x": inp["x"], "targets": t.to(ids)}
    if vocab is not None:
        p["w_emb"] = torch.randn(vocab, H, generator=g).to(torch.bfloat16)
        inp = {"targets": inp["targets"], "tokens": torch.randint(-1, vocab, (S,), generator=g).to(ids)}
    return inp, p


def run(S, Hq, Hkv, D, offsets, rotary, loss, vocab=None, ends=None, seed=0, drop=(7, 30), steps=1, **kw):
    announce(f"layer step S={S} offsets={offsets} {vars(rotary) if rotary else None} {vars(loss) if loss else None} "
             f"vocab={vocab} {kw}")
    classes = loss.classes if loss is not None else None
    inp, p = setup(S, Hq, Hkv, D, classes, vocab, seed, ends, kw.pop("ids", torch.int64))
    walk = {k: kw.pop(k) for k in ("lookahead", "poison", "loss_scale") if k in kw}
    rows = kw.pop("rows", None)
    lay = ChunkedLayer(S, len(offsets) - 1, Hq, Hkv, D, offsets=offsets, rotary=rotary, loss=loss, vocab=vocab,
                       ends=ends, **kw)
    if rows is not None:
        lay.set_offload_rows(rows)
    out = lay.alloc_outputs()
    dp = {k: v.cuda() for k, v in p.items()}
    for _ in range(steps):
        lay.step({k: v.cuda() for k, v in inp.items()}, dp, out, seed=drop[0], offset=drop[1], **walk)
    torch.cuda.synchronize()
    lay.close()
    return {k: to_np(v) for k, v in out.items()}, inp, p


def check(got, ref):
    assert set(got) == set(ref)
    for k in ref:
        g, r = got[k], ref[k]
        assert np.isfinite(g).all(), k
        rel = np.linalg.norm(g - r) / np.linalg.norm(r)
        mx = np.abs(g - r).max() / np.abs(r).max()
        print(f"  {k:8s} rel_fro {rel:.2e} max_rel {mx:.2e}", file=sys.stderr, flush=True)
        assert rel <= REL and mx <= MAXREL, (k, rel, mx)


def rope_of(rotary, D):
    o = dict(rotary.freqs)
    o["kind"] = o.pop("scaling", "none")
    rot = D if rotary.rot is None else rotary.rot
    freqs, amp = O.rope_freqs(rot, **o)
    return dict(rot=rot, layout=rotary.layout, freqs=freqs, amp=amp, position0=rotary.position0)


@pytest.mark.parametrize("Hq,Hkv,D,offsets,rotary,loss,vocab,ends", [
    (2, 2, 128, [0, 128, 256, 384, 512], Rotary(), Loss(512), None, None),
    (4, 2, 64, [0, 100, 101, 300, 512], Rotary(rot=32, layout="interleaved", position0=100000, scaling="yarn",
                                               factor=8.0, original_len=4096), Loss(256, 0.1, 1e-3), 200, None),
    (4, 2, 64, [0, 77, 300], Rotary(base=500000.0), Loss(768, 0.0, 1e-4), 50,
     BlockEnds("rms", True, 0.9, 0.7, 0.1)),
])
def test_layer_step_matches_oracle(Hq, Hkv, D, offsets, rotary, loss, vocab, ends):
    S, drop, scale = offsets[-1], (2 ** 60 + 5, 2 ** 33), 0.5
    got, inp, p = run(S, Hq, Hkv, D, offsets, rotary, loss, vocab, ends, seed=1, drop=drop, loss_scale=scale,
                      ids=torch.int32)
    H = Hq * D
    pr = ends.dropout if ends else 0.0
    keep = [T.keep_factor(S, H, pr, drop[0], drop[1] + site) for site in (C.DROP_EMBED, C.DROP_ATTN, C.DROP_MLP)]
    hp = {k: to_np(v) for k, v in p.items()}
    x = to_np(inp["x"]) if vocab is None else T.embedding_fwd(inp["tokens"].numpy(), hp["w_emb"], 1.0, keep[0])
    e = dict(norm=ends.norm, gate=ends.gate, alpha=ends.residual_scale, scale=ends.branch_scale) if ends else None
    hp.pop("w_emb", None)
    ref = O.layer_step(x, hp, Hq, Hkv, D, rope_of(rotary, D), inp["targets"].numpy(), loss.label_smoothing,
                       loss.z_loss, scale, e, keep[1:])
    if vocab is not None:
        ref["dw_emb"] = T.embedding_bwd(inp["tokens"].numpy(), ref.pop("dx"), vocab, 1.0, keep[0])
    check(got, ref)


@pytest.mark.parametrize("offload,rows", [("qol", None), ("qkvol", [200, 0, 1, 512]), ("qkvol_evict", None)])
def test_layer_step_offload_is_bitwise_invisible(offload, rows):
    offsets = [0, 256, 512, 768, 1024]
    if rows is not None:
        rows = [min(r, offsets[i + 1] - offsets[i]) for i, r in enumerate(rows)]
    kw = dict(rotary=Rotary(rot=64), loss=Loss(512), vocab=100, ends=BlockEnds("layer", True, 1.0, 0.5, 0.1), seed=2)
    base, _, _ = run(1024, 2, 2, 128, offsets, **kw)
    got, _, _ = run(1024, 2, 2, 128, offsets, **kw, offload=offload, poison=True, lookahead=1, rows=rows, steps=2)
    for k in base:
        assert np.array_equal(got[k], base[k]), k


def test_layer_rotary_depends_on_differences_only():
    """Another first position: the same outputs within the gates (the angles'
    roundings differ); without the rotation they differ by O(1)."""
    offsets = [0, 130, 256]
    a, _, _ = run(256, 2, 2, 128, offsets, Rotary(position0=0), Loss(256), seed=3)
    b, _, _ = run(256, 2, 2, 128, offsets, Rotary(position0=2 ** 40 + 3), Loss(256), seed=3)
    check(b, a)
    c, _, _ = run(256, 2, 2, 128, offsets, None, Loss(256), seed=3)
    assert np.linalg.norm(c["dw_qkv"] - a["dw_qkv"]) > 0.1 * np.linalg.norm(a["dw_qkv"])


def test_layer_rotary_with_given_frequencies():
    """A stretched context's frequencies and amplitude, given: what the scaling by
    name makes of them within the gates (the table's roundings differ); plain
    positions move the outputs by O(1)."""
    offsets = [0, 130, 256]
    named = Rotary(scaling="yarn", factor=8.0, original_len=32, beta_fast=4.0)
    rope = rope_of(named, 128)
    given = Rotary(inv_freq=[float(f) for f in rope["freqs"]], amp=rope["amp"])
    a, _, _ = run(256, 2, 2, 128, offsets, named, Loss(256), seed=3)
    b, _, _ = run(256, 2, 2, 128, offsets, given, Loss(256), seed=3)
    check(b, a)
    c, _, _ = run(256, 2, 2, 128, offsets, Rotary(), Loss(256), seed=3)
    assert np.linalg.norm(c["dw_qkv"] - a["dw_qkv"]) > 0.05 * np.linalg.norm(a["dw_qkv"])


def test_layer_loss_scale_on_the_device():
    offsets = [0, 130, 256]
    a, _, _ = run(256, 2, 2, 128, offsets, None, Loss(256), seed=4, loss_scale=0.125)
    b, _, _ = run(256, 2, 2, 128, offsets, None, Loss(256), seed=4, loss_scale=torch.tensor([0.125], device="cuda"))
    c, _, _ = run(256, 2, 2, 128, offsets, None, Loss(256), seed=4)  # 1 / S
    d, _, _ = run(256, 2, 2, 128, offsets, None, Loss(256), seed=4, loss_scale=1.0 / 256)
    for k in a:
        assert np.array_equal(a[k], b[k]) and np.array_equal(c[k], d[k]), k


def test_layer_step_refuses():
    lay = ChunkedLayer(256, 1, 2, 2, 128, loss=Loss(256), rotary=Rotary())
    out = lay.alloc_outputs()
    inp, p = setup(256, 2, 2, 128, 256, None, 1)
    t, x = inp["targets"].cuda(), inp["x"].cuda()
    dp = {k: v.cuda() for k, v in p.items()}
    for bad in (t[:255], t.to(torch.int16), t.repeat(2)[::2], inp["targets"]):
        with pytest.raises(ValueError):
            lay.step({"x": x, "targets": bad}, dp, out)
    for bad in (float("inf"), float("nan"), torch.ones(2, device="cuda"), torch.ones(1),
                torch.ones(1, device="cuda").double()):
        with pytest.raises(ValueError):
            lay.step({"x": x, "targets": t}, dp, out, loss_scale=bad)
    lay.close()
    with pytest.raises(ValueError):
        ChunkedLayer(2 ** 15, 1, 2, 2, 128, loss=Loss(2 ** 16))


# --------------------------------------------------------------------- training
class Training:
    """A layer from tokens to its loss with an optimizer over all parameters."""

    def __init__(self, state, seed=5, max_norm=0.5, **opt):
        S, Hq, Hkv, D, self.vocab = 256, 2, 1, 128, 96
        self.offsets = [0, 100, 256]
        self.rotary, self.loss = Rotary(), Loss(256)
        inp, p = setup(S, Hq, Hkv, D, 256, self.vocab, seed)
        self.inp, self.p = ({k: v.cuda() for k, v in d.items()} for d in (inp, p))
        # The packed projection needs (Hq + 2 Hkv) D to be a multiple of 256.
        self.lay = ChunkedLayer(S, 2, Hq, Hkv, D, offsets=self.offsets, rotary=self.rotary, loss=self.loss,
                                vocab=self.vocab)
        self.out = self.lay.alloc_outputs()
        self.opt = AdamW(self.p, {k: self.out["d" + k] for k in self.p}, lr=3e-3, max_norm=max_norm, state=state,
                         lr_scale={"w_emb": 2.0}, seed=9, **opt)

    def step(self):
        self.lay.step(self.inp, self.p, self.out, loss_scale=1.0 / 256)
        self.opt.step()
        return self.out["loss"].mean().item()


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_training_steps(state):
    """Steps of the layer with its optimizer, each update against the oracle's
    from the gradients and states before it: the norm to fp32's half step, the
    parameters to the roundings that test_gpu_step_ops.py counts (with the
    8-bit states' decoded values)."""
    announce(f"training {state}")
    k = Training(state)
    u = 2.0 ** -24
    for t in (1, 2, 3):
        k.lay.step(k.inp, k.p, k.out, loss_scale=1.0 / 256)
        s = {n: v.cpu().numpy().copy() for n, v in k.opt.state_tensors().items()}
        old = {n: to_np(k.opt.master.get(n, k.p[n])) for n in k.p}
        k.opt.step()
        norm, f = O.grad_norm([to_np(g) for g in k.opt.grads.values()], 0.5)
        got = to_np(k.opt.norm)
        assert abs(got[0] - norm) <= 1.01 * u * norm and abs(got[1] - f) <= 2.1 * u * f and k.opt.steps.item() == t
        for n, p in k.p.items():
            if state == "f32":
                m, v = s["m." + n], s["v." + n]
            else:
                m = O.value8(s["m." + n], s["m_scale." + n])
                v = O.value8(s["v." + n], s["v_scale." + n]) ** 2
            w, g = old[n].ravel(), to_np(k.opt.grads[n]).ravel()
            lr, wd = 3e-3 * (2.0 if n == "w_emb" else 1.0), 0.1 if p.dim() >= 2 else 0.0
            rp, rm, rv = O.adamw(w, g, m, v, t, lr, 0.9, 0.95, 1e-8, wd, float(got[1]))
            tm = 4 * u * (0.9 * np.abs(m) + 0.1 * np.abs(got[1] * g)) + 2.0 ** -148
            den = np.sqrt(rv / (1 - 0.95 ** t)) + 1e-8
            q = rm / (1 - 0.9 ** t) / den
            tol = lr * (tm / (1 - 0.9 ** t) / den + 12 * u * np.abs(q) + 4 * u * (np.abs(q) + np.abs(wd * w))) \
                + 2 * u * np.abs(w)
            now = to_np(k.opt.master.get(n, p)).ravel()
            assert (np.abs(now - rp) <= tol).all(), (n, np.abs(now - rp).max())
            if n in k.opt.master:
                assert torch.equal(p, k.opt.master[n].view_as(p).to(torch.bfloat16)), n
    k.lay.close()


def test_training_resumes_from_its_state():
    """A second run that copies the first's parameters and state goes on with the
    same bits; an update under an infinite gradient changes nothing."""
    announce("training resumes")
    a, b = Training("e4m3"), Training("e4m3", seed=6)
    b.inp = a.inp
    for _ in range(2):
        a.step()
    for n, t in b.p.items():
        t.copy_(a.p[n])
    for n, t in b.opt.state_tensors().items():
        t.copy_(a.opt.state_tensors()[n])
    for _ in range(2):
        a.step()
        b.step()
    for n in a.p:
        assert torch.equal(a.p[n], b.p[n]), n
    a.out["dw_o"][3, 3] = float("inf")
    kept = {n: t.clone() for n, t in a.opt.state_tensors().items()}
    a.opt.step()
    for n, t in a.opt.state_tensors().items():
        assert torch.equal(t, kept[n]), n
    for n in a.p:
        assert torch.equal(a.p[n], b.p[n]), n
    a.lay.close()
    b.lay.close()


def test_optimizer_on_another_stream_and_in_a_graph():
    """step() with a stream, and captured with a device learning rate: the bits of
    eager steps with the same numbers."""
    announce("optimizer in a graph")

    def make():
        g = torch.Generator().manual_seed(1)
        p = {"w": torch.randn(300, 7, generator=g).to(torch.bfloat16).cuda(), "b": torch.randn(5, generator=g).cuda()}
        d = {k: torch.randn(v.shape, generator=g).cuda() for k, v in p.items()}
        return AdamW(p, d, lr=1e-2, max_norm=1.0, state="e4m3", seed=3)

    a, b, c = make(), make(), make()
    lrs = [1e-2, 5e-3, 1e-3]
    for lr in lrs:
        a.step(lr)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for lr in lrs:
        b.step(lr, stream=s)
    lr = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    s2 = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s2):
        c.step(lr)
    for x in lrs:
        lr.fill_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        torch.randn(100, device="cuda").sum().item()
    for o in (b, c):
        for n, t in o.state_tensors().items():
            assert torch.equal(t, a.state_tensors()[n]), n
        for n in a.params:
            assert torch.equal(o.params[n], a.params[n]), n


def test_optimizer_refuses():
    p, g = {"w": torch.zeros(8, 8, device="cuda")}, {"w": torch.zeros(8, 8, device="cuda")}
    for params, grads in (({"w": p["w"].half()}, g), (p, {"w": g["w"].t()[:, :4]}), (p, {"w": g["w"][:4]}),
                          ({"w": p["w"].t()[1:]}, g), (p, {"w": g["w"].cpu()})):
        with pytest.raises(ValueError):
            AdamW(params, grads, 1e-3)
    with pytest.raises(ValueError):
        AdamW(p, g, 1e-3, lr_scale={"v": 1.0})
    o = AdamW(p, g, 1e-3)
    for lr in (torch.ones(1), torch.ones(2, device="cuda"), torch.ones(1, device="cuda").double(), INF, float("nan")):
        with pytest.raises(ValueError):
            o.step(lr)
    assert o.steps.item() == 0


def test_optimizer_counts_no_update_that_is_refused():
    """Settings that are changed between steps to what the update's call refuses:
    nothing is enqueued and nothing counted."""
    announce("optimizer with settings that are refused")
    p, g = {"w": torch.ones(8, 8, device="cuda")}, {"w": torch.ones(8, 8, device="cuda")}
    o = AdamW(p, g, 1e-3)
    o.step()
    kept = {n: t.clone() for n, t in o.state_tensors().items()}
    for name, bad in (("eps", 1e-40), ("eps", INF), ("eps", 0.0), ("betas", (0.9, 1.0)), ("betas", (0.9,)),
                      ("seed", 0.5), ("lr", INF), ("lr", torch.ones(1)), ("max_norm", 0.0)):
        good = getattr(o, name)
        setattr(o, name, bad)
        with pytest.raises((ValueError, TypeError, L.SppoError)):
            o.step()
        setattr(o, name, good)
        for n, t in o.state_tensors().items():
            assert torch.equal(t, kept[n]), (name, bad, n)
    o.step()
    assert o.steps.item() == 2


def test_optimizer_steps_at_once_on_another_stream(monkeypatch):
    """The first step() on a stream that waits for nothing, while the
    constructor's stream is still busy with what was enqueued after the list's
    table: state, norm and count are ready by then."""
    announce("optimizer at once on another stream")
    real = L.opt_list

    def busy(*a):
        out = real(*a)
        torch.cuda._sleep(10 ** 8)  # some 40 ms before whatever the constructor fills after this
        return out

    monkeypatch.setattr(L, "opt_list", busy)
    g = torch.Generator().manual_seed(1)
    p0 = torch.randn(300, 7, generator=g).cuda()
    grad = {"w": torch.randn(300, 7, generator=g).cuda()}
    torch.cuda.synchronize()
    for state in ("f32", "e4m3"):
        params = [{"w": p0.clone()} for _ in range(2)]
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        a = AdamW(params[0], grad, lr=1e-2, max_norm=1.0, state=state)
        a.step(stream=s)
        torch.cuda.synchronize()
        b = AdamW(params[1], grad, lr=1e-2, max_norm=1.0, state=state)
        torch.cuda.synchronize()
        b.step()
        torch.cuda.synchronize()
        assert a.steps.item() == 1 and torch.equal(a.norm, b.norm)
        for n, t in a.state_tensors().items():
            assert torch.equal(t, b.state_tensors()[n]), n
        assert torch.equal(params[0]["w"], params[1]["w"])


def test_layer_with_a_loss_steps_at_once_on_another_stream():
    """A first step on a stream that waits for nothing, while the stream that the
    layer was made on was busy: the bits of a step that waited."""
    announce("layer at once on another stream")
    inp, p = setup(256, 2, 2, 128, 256, None, 1)
    inp, p = ({k: v.cuda() for k, v in d.items()} for d in (inp, p))
    outs = []
    for busy in (True, False):
        made, s = torch.cuda.Stream(), torch.cuda.Stream()
        with torch.cuda.stream(made):
            # What the layer's buffers may be made of holds no zeros.
            old = [torch.full((256, 256), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(64)]
            made.synchronize()
            del old
            if busy:
                torch.cuda._sleep(10 ** 8)  # some 40 ms
            lay = ChunkedLayer(256, 2, 2, 2, 128, offsets=[0, 100, 256], loss=Loss(256), rotary=Rotary())
            out = lay.alloc_outputs()
        if not busy:
            torch.cuda.synchronize()
        lay.step(inp, p, out, stream=s)
        torch.cuda.synchronize()
        outs.append({k: v.clone() for k, v in out.items()})
        lay.close()
    for k in outs[0]:
        assert torch.isfinite(outs[0][k].float()).all() and torch.equal(outs[0][k], outs[1][k]), k
