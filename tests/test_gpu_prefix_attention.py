"""sf_op_prefix_attention against its definition in doubles: head layouts, lengths from one key on, ends inside a tile, dead slots
that hold NaN, rising scores, capture, streams.

Tolerances.  With A = sum_j p_j |v_j| of a row, bf16 mode rounds every p_j once (2^-8 of it: 2^-8 A) and the output once
(2^-8 |o|); a score is a float sum of hd products, off by (hd + 4) 2^-24 sum |q k| scale, and the softmax takes it twice (its
numerator and its sum); sums of n terms in float are off by n 2^-24."""
import numpy as np
import pytest
import torch

from paper_2511_20340_amd import binding as sfb
from paper_2511_20340_amd.engine import Engine

pytestmark = pytest.mark.gpu

HEADS = {"f32": (4, 4, 64, "f32"), "f32-gqa-hd24": (8, 2, 24, "f32"), "1b": (32, 8, 64, "bf16"), "8b": (32, 8, 128, "bf16"),
         "14b": (40, 8, 128, "bf16"), "one-head": (1, 1, 64, "bf16"), "mqa": (12, 1, 128, "bf16"), "3-kv": (3, 3, 128, "bf16")}


def make(heads, B, n_q, P, cap, seed, pcap=None):
    hq, hkv, hd, dtype = HEADS[heads]
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    cfg = {"n_layers": 1, "d_model": 64, "n_q_heads": hq, "n_kv_heads": hkv, "head_dim": hd, "d_ffn": 64, "vocab": 64, "dtype": dtype}
    pcap = pcap or max(32, -(-P // 32) * 32)
    eng, one = Engine(cfg, B, cap, n_q - 1), Engine(cfg, 1, pcap, 0)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(t)  # noqa: E731
    return eng, one, r(B, n_q, hq, hd), r(1, hkv, pcap, hd), r(1, hkv, pcap, hd), r(B, hkv, cap, hd), r(B, hkv, cap, hd)


def load(eng, one, pk, pv, k, v):
    one.sf_kv_import(pk, "tk"); one.sf_kv_import(pv, "tv"); eng.sf_kv_import(k, "tk"); eng.sf_kv_import(v, "tv")


def call(eng, one, q, P, lens, n_q, mask, upper=None):
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return eng.sf_op_prefix_attention(q, one.layer_cache("tk"), one.layer_cache("tv"), P, eng.layer_cache("tk"),
                                      eng.layer_cache("tv"), kv, n_q, mask, len_upper=max(lens) if upper is None else upper)


def check(got, q, pk, pv, k, v, P, lens, mask, bf16):
    B, n_q, hq, hd = q.shape
    hkv = k.shape[1]
    G, worst = hq // hkv, 0.0
    for b in range(B):
        for g in range(hkv):
            heads = slice(g * G, (g + 1) * G)
            K = torch.cat([pk[0, g, :P], k[b, g, :lens[b] + n_q]]).double()
            V = torch.cat([pv[0, g, :P], v[b, g, :lens[b] + n_q]]).double()
            Q = q[b, :, heads].double()                                     # [n_q, G, hd]
            s = Q @ K.t() * hd ** -0.5
            size = (Q.abs() @ K.abs().t() * hd ** -0.5).amax(-1, keepdim=True)
            j = torch.arange(K.shape[0], device="cuda") - P - lens[b]
            if mask == sfb.SF_MASK_CAUSAL:
                hidden = j[None, :] > torch.arange(n_q, device="cuda")[:, None]
                s = s.masked_fill(hidden[:, None], -float("inf"))
            p = torch.softmax(s, -1)
            want, A = p @ V, p @ V.abs()
            tol = A * (2 * (hd + 4) * 2.0 ** -24 * size + (K.shape[0] + 32) * 2.0 ** -24) + 1e-30
            if bf16:
                tol = tol + 2.0 ** -8 * A + 2.0 ** -8 * want.abs()
            err = (got[b, :, heads].double() - want).abs()
            worst = max(worst, float((err / tol).max()))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("mask", [sfb.SF_MASK_CAUSAL, sfb.SF_MASK_BIDIR])
@pytest.mark.parametrize("heads,B,n_q", [("f32", 3, 5), ("f32-gqa-hd24", 2, 3), ("1b", 1, 1), ("1b", 3, 5), ("8b", 2, 9), ("8b", 33, 1),
                                         ("14b", 7, 5), ("14b", 1, 7), ("one-head", 5, 1), ("one-head", 1, 40), ("mqa", 3, 20),
                                         ("3-kv", 4, 3)])
@pytest.mark.parametrize("P", [1, 31, 32, 33, 64, 65, 300, 1031])
def test_against_the_definition(heads, B, n_q, P, mask):
    cap = 256
    eng, one, q, pk, pv, k, v = make(heads, B, n_q, P, cap, P * 10 + n_q)
    rng = np.random.default_rng(P + B)
    lens = [int(x) for x in rng.integers(0, cap - n_q + 1, size=B)]
    lens[0] = 0
    lens[-1] = [0, 1, 27, 32, cap - n_q][P % 5]
    # what no row may see holds NaN: the prefix behind its end, the own caches behind the block
    pk2, pv2, k2, v2 = pk.clone(), pv.clone(), k.clone(), v.clone()
    pk2[:, :, P:], pv2[:, :, P:] = float("nan"), float("nan")
    for b in range(B):
        k2[b, :, lens[b] + n_q:], v2[b, :, lens[b] + n_q:] = float("nan"), float("nan")
    load(eng, one, pk2, pv2, k2, v2)
    got = call(eng, one, q, P, lens, n_q, mask)
    check(got, q, pk, pv, k, v, P, lens, mask, HEADS[heads][3] == "bf16")


@pytest.mark.parametrize("heads,B,n_q,P,cap", [("14b", 60, 5, 4100, 320), ("1b", 100, 2, 2500, 64), ("8b", 2, 1, 20000, 1024),
                                               ("8b", 1, 5, 700, 8192)])
def test_large(heads, B, n_q, P, cap):
    eng, one, q, pk, pv, k, v = make(heads, B, n_q, P, cap, 7)
    lens = [int(x) for x in np.random.default_rng(3).integers(0, cap - n_q + 1, size=B)]
    lens[0] = cap - n_q
    load(eng, one, pk, pv, k, v)
    got = call(eng, one, q, P, lens, n_q, sfb.SF_MASK_CAUSAL)
    pick = [0, B // 2, B - 1] if B > 3 else list(range(B))
    check(got[pick], q[pick], pk, pv, k[pick], v[pick], P, [lens[b] for b in pick], sfb.SF_MASK_CAUSAL, True)


@pytest.mark.parametrize("heads", ["f32", "1b", "14b"])
@pytest.mark.parametrize("order", ["rising", "falling", "one key", "far apart"])
def test_scores_that_move_the_maximum(heads, order):
    """Along the prefix the scores rise or fall by hundreds, one key outweighs all, or all lie far from zero."""
    B, n_q, P, cap = 3, 2, 500, 64
    eng, one, q, pk, pv, k, v = make(heads, B, n_q, P, cap, 11)
    hd = q.shape[-1]
    q = torch.sign(q) * 0 + 1
    ramp = torch.linspace(-1, 1, pk.shape[2], device="cuda")
    step = {"rising": ramp * 12, "falling": -ramp * 12, "one key": torch.where(torch.arange(pk.shape[2], device="cuda") == 77, 6.0, -6.0),
            "far apart": torch.where(torch.arange(pk.shape[2], device="cuda") % 3 == 0, 40.0, -40.0)}[order]
    pk = (step[None, None, :, None] + torch.zeros_like(pk, dtype=torch.float32)).to(pk.dtype)
    pk[..., hd // 2:] *= 0.5
    lens = [5, 0, 30]
    load(eng, one, pk, pv, k, v)
    got = call(eng, one, q.contiguous(), P, lens, n_q, sfb.SF_MASK_CAUSAL)
    assert torch.isfinite(got.float()).all()
    check(got, q, pk, pv, k, v, P, lens, sfb.SF_MASK_CAUSAL, HEADS[heads][3] == "bf16")


@pytest.mark.parametrize("heads", ["f32", "8b"])
def test_no_prefix_is_the_attention_without(heads):
    eng, one, q, pk, pv, k, v = make(heads, 3, 4, 32, 96, 5)
    load(eng, one, pk, pv, k, v)
    lens = [10, 0, 77]
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = eng.sf_op_attention(q, eng.layer_cache("tk"), eng.layer_cache("tv"), kv, 4, sfb.SF_MASK_BIDIR)
    assert torch.equal(call(eng, one, q, 0, lens, 4, sfb.SF_MASK_BIDIR), want)


@pytest.mark.parametrize("heads", ["f32", "14b"])
def test_a_loose_bound_and_repeats(heads):
    """A bound above the lengths changes nothing but the split; the same call has the same bits."""
    eng, one, q, pk, pv, k, v = make(heads, 4, 3, 200, 2048, 6)
    load(eng, one, pk, pv, k, v)
    lens = [3, 700, 41, 0]
    a = call(eng, one, q, 200, lens, 3, sfb.SF_MASK_CAUSAL)
    assert torch.equal(a, call(eng, one, q, 200, lens, 3, sfb.SF_MASK_CAUSAL))
    b = call(eng, one, q, 200, lens, 3, sfb.SF_MASK_CAUSAL, upper=2048 - 3)
    for x in (a, b):
        check(x, q, pk, pv, k, v, 200, lens, sfb.SF_MASK_CAUSAL, HEADS[heads][3] == "bf16")


def test_captured_and_on_another_stream():
    eng, one, q, pk, pv, k, v = make("8b", 6, 2, 900, 128, 8)
    load(eng, one, pk, pv, k, v)
    lens = [0, 5, 100, 64, 31, 126]
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    run = lambda: eng.sf_op_prefix_attention(q, one.layer_cache("tk"), one.layer_cache("tv"), 900, eng.layer_cache("tk"),  # noqa: E731
                                             eng.layer_cache("tv"), kv, 2, sfb.SF_MASK_CAUSAL, len_upper=126)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run()
    torch.cuda.synchronize()
    assert torch.equal(other, run())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for it in range(4):
        q.normal_()
        kv.copy_(torch.tensor(lens[it:] + lens[:it], dtype=torch.int32))
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), it
