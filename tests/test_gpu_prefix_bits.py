"""What a row over a shared prefix does not depend on, to the last bit: the scores of the rows beside it, the length of the block
that it is verified in, the part of the batch that runs."""
import numpy as np
import pytest
import torch

import synth
from paper_2511_20340_amd import binding as sfb
from paper_2511_20340_amd import engine as E

from test_gpu_e2e import SLICES
from test_gpu_prefix_attention import call, load, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", ["f32", "1b", "8b", "14b"])
@pytest.mark.parametrize("B,n_q", [(3, 2), (7, 5)])
def test_a_row_does_not_hang_on_its_neighbours(heads, B, n_q):
    """The other sequences' scores rise and fall by hundreds along the prefix; one sequence keeps its bits, wherever it stands."""
    P, cap = 700, 64
    eng, one, q, pk, pv, k, v = make(heads, B, n_q, P, cap, 21)
    ramp = torch.linspace(-1, 1, pk.shape[2], device="cuda")[None, None, :, None]
    pk = (pk.float() * 0.5 + ramp * torch.where(torch.arange(q.shape[-1], device="cuda") % 2 == 0, 1.0, -0.5)).to(pk.dtype)
    load(eng, one, pk, pv, k, v)
    lens = [20] * B
    for b in (0, B // 2, B - 1):
        want = call(eng, one, q, P, lens, n_q, sfb.SF_MASK_CAUSAL)[b].clone()
        for scale in (0.0, 4.0, -4.0, 50.0):
            other = q * scale
            other[b] = q[b]
            got = call(eng, one, other, P, lens, n_q, sfb.SF_MASK_CAUSAL)[b]
            assert torch.equal(got, want), (b, scale)


def engines(shape, B, cap, k, seed, P, n=1):
    tw, dw = synth.target_weights(shape, seed, 0.05), synth.draft_weights(shape, k, seed, 0.05)
    one = E.Engine(shape.cfg(), 1, -(-(P + 8) // 32) * 32, 3)
    one.bind(tw, dw)
    one.prefill(synth.prompts([P], shape.vocab, seed), block=64)
    out = [E.Engine(shape.cfg(), B, cap, k) for _ in range(n)]
    for e in out:
        e.bind(tw, dw)
        e.sf_set_prefix(one)
    return one, out


@pytest.mark.parametrize("name,B,P,tail", [("8b-slice", 12, 1000, 10), ("1b-slice", 12, 1500, 40), ("14b-slice", 5, 900, 600)])
def test_one_engine_switching_between_plain_and_speculative_steps(name, B, P, tail):
    """Plain greedy steps (k = 0) and a verified block (k = 4) of one engine give the same logits for the same rows: over the
    prefix alone and over tails of their own, short and of several chunks."""
    m, k, seed = SLICES[name], 4, 23
    cap = -(-(tail + 4 * (k + 1)) // 32) * 32
    _, (eng,) = engines(m, B, cap, k, seed, P)
    none = torch.zeros(B, 0, dtype=torch.int32, device="cuda")
    for start in ("prefix", "tails"):
        if start == "tails":
            eng.prefill(synth.prompts([max(1, tail - 3 * b) for b in range(B)], m.vocab, seed + 1), block=16)
        else:
            eng.pending.copy_(torch.arange(B, device="cuda") * 17 + 3)    # sequences that differ
        snap = {n: getattr(eng, n).clone() for n in ("kv_len", "pending", "n_new", "cu_new", "hooks")}
        len0 = eng.len_upper
        toks, rows = [eng.pending.clone()], []
        for _ in range(k + 1):
            lg, ids = eng.sf_verify_step(0, none)
            rows.append(lg[:, 0].clone())
            _, out = eng.sf_accept_commit(0, none, ids)
            toks.append(out[:, 0].clone())
        for n, t in snap.items():
            getattr(eng, n).copy_(t)
        eng.len_upper = len0
        draft = torch.stack(toks[1:k + 1], 1).contiguous()
        lg, ids = eng.sf_verify_step(k, draft)
        for i in range(k + 1):
            assert torch.equal(lg[:, i], rows[i]), (start, i)
        acc, _ = eng.sf_accept_commit(k, draft, ids)
        assert acc.cpu().tolist() == [k + 1] * B, start


@pytest.mark.parametrize("name,block,lens,P", [("8b-slice", 16, [1, 15, 16, 17, 40, 40, 3, 64], 1500), ("1b-slice", 8, [5, 30, 8, 8, 9], 1500),
                                               ("14b-slice", 32, [700, 1, 33, 580], 900)])
def test_packed_prefill_keeps_the_whole_batchs_bits(name, block, lens, P):
    """Tails prefilled over the prompts that have started leave what running all of them in every block leaves."""
    m, k, seed, B = SLICES[name], 4, 29, len(lens)
    cap = -(-(max(lens) + block + k) // 32) * 32
    one, (eng, ref) = engines(m, B, cap, k, seed, P, n=2)
    prompts = synth.prompts(lens, m.vocab, seed + 2)
    first = eng.prefill(prompts, block=block)
    helper = E.Engine(ref.cfg, B, cap, block - 1, share_caches=ref)
    helper.bind_shared(ref, with_draft=True)
    helper.sf_set_prefix(one, start=False)
    want = E._prefill_blocks(helper, prompts, block, k)
    torch.cuda.synchronize()
    assert eng.kv_len.tolist() == lens
    for which, layers in (("tk", m.n_layers), ("tv", m.n_layers), ("dk", 1), ("dv", 1)):
        for l in range(layers):
            a, b = eng.sf_kv_export(which, l), ref.sf_kv_export(which, l)
            for i in range(B):
                assert torch.equal(a[i, :, :lens[i]], b[i, :, :lens[i]]), (which, l, i)
    rows = helper.hooks[torch.arange(B), (helper.n_new.long() - 1).cpu()]
    assert torch.equal(eng.hooks[:, 0], rows) and torch.equal(first, want)
