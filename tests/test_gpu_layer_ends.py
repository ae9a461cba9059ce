"""The chunked layer with the training operators around its blocks: tokens in
(embedding, its gradient summed over the reverse walk), norms after the
branches, gates, scales and dropout, against the fp64 oracle; the masks and
results do not depend on the chunking or on what is offloaded.

Gates as in test_gpu_layer.py (bf16 activations at every step): per tensor,
relative Frobenius error <= 1.2e-2 and max |err| <= 1.5e-2 of max |ref|; the
block ends round no more often than the adds that they replace, and the
embedding adds one rounding.  A mask drawn at another place, a missing gate or
scale moves its outputs by O(1).
"""
import sys

import numpy as np
import pytest
import torch

from oracle import train_ops as O
from paper_2503_10377_amd import chunked_layer as C
from paper_2503_10377_amd.chunked_layer import BlockEnds, ChunkedLayer
from paper_2503_10377_amd.inputs import make_layer_inputs
from parity import to_np

pytestmark = pytest.mark.gpu
REL, MAXREL = 1.2e-2, 1.5e-2


def announce(msg):
    print(f"\n[case] {msg}", file=sys.stderr, flush=True)


def setup(S, Hq, Hkv, D, ends, vocab, seed, id_dtype=torch.int64):
    inp, p = make_layer_inputs(S, Hq, Hkv, D, seed, device="cpu")
    H = Hq * D
    g = torch.Generator().manual_seed(1000 + seed)
    for n in (1, 2):
        for k, name in ends.params(n).items() if ends is not None else ():
            r = torch.randn(H, generator=g)
            p[name] = 0.1 * r if k == "post_beta" else 1.0 + 0.1 * r
    if vocab is not None:
        p["w_emb"] = torch.randn(vocab, H, generator=g).to(torch.bfloat16)
        ids = torch.randint(-1, vocab, (S,), generator=g)
        ids[::7] = 3  # a frequent token
        inp = {"dy": inp["dy"], "tokens": ids.to(id_dtype)}
    return inp, p


def run(S, Hq, Hkv, D, offsets, ends, vocab, seed=0, drop=(7, 30), steps=1, **kw):
    announce(f"layer with ends S={S} offsets={offsets} vocab={vocab} "
             f"{vars(ends) if ends is not None else None} {kw}")
    inp, p = setup(S, Hq, Hkv, D, ends, vocab, seed, kw.pop("id_dtype", torch.int64))
    walk = {k: kw.pop(k) for k in ("lookahead", "poison") if k in kw}
    rows = kw.pop("rows", None)
    lay = ChunkedLayer(S, len(offsets) - 1, Hq, Hkv, D, offsets=offsets, ends=ends, vocab=vocab,
                       embed_scale=0.5 if vocab is not None else 1.0, **kw)
    if rows is not None:
        lay.set_offload_rows(rows)
    out = lay.alloc_outputs()
    dp = {k: v.cuda() for k, v in p.items()}
    for _ in range(steps):
        lay.step({k: v.cuda() for k, v in inp.items()}, dp, out, seed=drop[0], offset=drop[1], **walk)
    torch.cuda.synchronize()
    lay.close()
    return {k: to_np(v) for k, v in out.items()}, inp, p


def oracle(S, Hq, Hkv, D, ends, vocab, inp, p, drop):
    H = Hq * D
    keep = [O.keep_factor(S, H, ends.dropout if ends else 0.0, drop[0], drop[1] + site)
            for site in (C.DROP_EMBED, C.DROP_ATTN, C.DROP_MLP)]
    hp = {k: to_np(v) for k, v in p.items()}
    x = to_np(inp["x"]) if vocab is None else O.embedding_fwd(inp["tokens"].numpy(), hp["w_emb"], 0.5, keep[0])
    e = dict(norm=ends.norm, gate=ends.gate, alpha=ends.residual_scale, scale=ends.branch_scale)
    ref = O.layer_with_ends(x, to_np(inp["dy"]), hp, Hq, Hkv, D, e, keep[1], keep[2])
    if vocab is not None:
        ref["dw_emb"] = O.embedding_bwd(inp["tokens"].numpy(), ref.pop("dx"), vocab, 0.5, keep[0])
    return ref


def check(got, ref):
    assert set(got) == set(ref)
    for k in ref:
        g, r = got[k], ref[k]
        assert np.isfinite(g).all(), k
        rel = np.linalg.norm(g - r) / np.linalg.norm(r)
        mx = np.abs(g - r).max() / np.abs(r).max()
        print(f"  {k:8s} rel_fro {rel:.2e} max_rel {mx:.2e}", file=sys.stderr, flush=True)
        assert rel <= REL and mx <= MAXREL, (k, rel, mx)


@pytest.mark.parametrize("Hq,Hkv,D,offsets,ends,vocab", [
    (2, 2, 128, [0, 128, 256, 384, 512], BlockEnds("layer", True, 0.9, 0.7, 0.1), 50),
    (4, 2, 64, [0, 100, 101, 300, 512], BlockEnds("rms", False, 1.0, 0.5, 0.2), 200),
    (4, 4, 64, [0, 77, 300], BlockEnds("none", False, 1.0, 1.0, 0.1), None),   # dropout alone
    (2, 2, 128, [0, 200, 256], BlockEnds("none", True, 1.0, 1.0, 0.0), 33),    # gates alone
])
def test_layer_with_ends_matches_oracle(Hq, Hkv, D, offsets, ends, vocab):
    S, drop = offsets[-1], (2 ** 60 + 5, 2 ** 33)
    got, inp, p = run(S, Hq, Hkv, D, offsets, ends, vocab, seed=1, drop=drop, id_dtype=torch.int32)
    check(got, oracle(S, Hq, Hkv, D, ends, vocab, inp, p, drop))


@pytest.mark.parametrize("offload,rows", [("qol", None), ("qkvol", [200, 0, 1, 512]), ("qkvol_evict", None)])
def test_layer_with_ends_offload_is_bitwise_invisible(offload, rows):
    offsets = [0, 256, 512, 768, 1024]
    if rows is not None:
        rows = [min(r, offsets[i + 1] - offsets[i]) for i, r in enumerate(rows)]
    ends = BlockEnds("layer", True, 1.0, 0.5, 0.1)
    base, _, _ = run(1024, 2, 2, 128, offsets, ends, 100, seed=2)
    got, _, _ = run(1024, 2, 2, 128, offsets, ends, 100, seed=2, offload=offload, poison=True, lookahead=1, rows=rows,
                    steps=2)
    for k in base:
        assert np.array_equal(got[k], base[k]), k


def test_layer_with_plain_ends_is_close_to_the_layer():
    """Ends that do nothing (scales of one, no norm, gate or dropout) against
    the layer without them: the same values but for one more rounding of each
    branch (the add then reads bf16), within the layer's gates."""
    offsets = [0, 130, 256]
    base, _, _ = run(256, 2, 2, 128, offsets, None, None, seed=3)
    got, _, _ = run(256, 2, 2, 128, offsets, BlockEnds(), None, seed=3)
    check(got, base)


def test_layer_with_ends_refuses():
    with pytest.raises(ValueError):
        BlockEnds("batch")
    with pytest.raises(ValueError):
        BlockEnds(dropout=1.0)
    with pytest.raises(ValueError):
        ChunkedLayer(256, 1, 2, 2, 128, vocab=0)
    lay = ChunkedLayer(256, 1, 2, 2, 128, vocab=10)
    out = lay.alloc_outputs()
    inp, p = setup(256, 2, 2, 128, None, 10, 1)
    t = inp["tokens"].cuda()
    # too short, another type, with gaps, in host memory
    for bad in (t[:255], t.to(torch.int16), t.repeat(2)[::2], inp["tokens"]):
        with pytest.raises(ValueError):
            lay.step({"tokens": bad, "dy": inp["dy"].cuda()}, {k: v.cuda() for k, v in p.items()}, out)
    lay.close()
