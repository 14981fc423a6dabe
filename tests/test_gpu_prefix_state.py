"""What a context and an engine know about a shared prefix: calls in another order, a prefix whose draft keys are not there,
sequences without a tail, memory that the steps still use."""
import pytest
import torch

import synth
from paper_2511_20340_amd import binding as sfb
from paper_2511_20340_amd.engine import Engine

from test_gpu_e2e import SLICES

pytestmark = pytest.mark.gpu
SHAPES = {"tiny": (synth.TINY, 0.02), "8b-slice": (SLICES["8b-slice"], 0.05)}


def weights(name, k, seed):
    shape, std = SHAPES[name]
    return shape, synth.target_weights(shape, seed, std), synth.draft_weights(shape, k, seed, std)


def test_a_block_verified_over_another_prefix_is_not_committed():
    k, seed, B = 2, 5, 2
    shape, tw, dw = weights("tiny", k, seed)
    one, eng = Engine(shape.cfg(), 1, 64, k), Engine(shape.cfg(), B, 64, k)
    for e in (one, eng):
        e.bind(tw, dw)
    one.prefill(synth.prompts([20], shape.vocab, seed))
    draft = torch.ones(B, k, dtype=torch.int32, device="cuda")
    for new in (one, one, None):
        _, ids = eng.sf_verify_step(k, draft)
        eng.sf_set_prefix(new)
        before = eng.kv_len.clone()
        with pytest.raises(sfb.SfError) as e:
            eng.sf_accept_commit(k, draft, ids)
        assert e.value.status == sfb.SF_ESTATE and torch.equal(eng.kv_len, before)
    _, ids = eng.sf_verify_step(k, draft)
    with pytest.raises(ValueError):
        eng.sf_set_prefix(one, length=0)                     # refused: the block stays
    eng.sf_accept_commit(k, draft, ids)


def logits_of_a_draft(eng, k):
    dl = torch.empty(eng.B, k, eng.V, device="cuda")
    eng.sf_draft_step(k, logits_out=dl)
    return dl


@pytest.mark.parametrize("name", SHAPES)
def test_a_prefix_taken_straight_after_a_commit(name):
    """The rows of the newest block get their draft keys before the prefix stands in front of anyone."""
    k, seed, B, P = 3, 7, 3, 40
    shape, tw, dw = weights(name, k, seed)
    got = []
    for drafted in (True, False):
        one, eng = Engine(shape.cfg(), 1, 64, k), Engine(shape.cfg(), B, 64, k)
        for e in (one, eng):
            e.bind(tw, dw)
        one.prefill(synth.prompts([P], shape.vocab, seed))
        draft = one.sf_draft_step(k)
        _, ids = one.sf_verify_step(k, draft)
        one.sf_accept_commit(k, ids[:, :k].contiguous(), ids)             # all of the block
        assert one.kv_len.tolist() == [P + k + 1]
        if drafted:
            one.sf_draft_step(k)
        eng.sf_set_prefix(one)
        assert one.kv_len.tolist() == [P + k + 1] and one.n_new.tolist() == [k + 1]
        got.append(logits_of_a_draft(eng, k))
    assert torch.equal(got[0], got[1])


def prefixes_without_draft_keys(shape, tw, dw, k, seed):
    prompt = synth.prompts([30], shape.vocab, seed)
    target_only = Engine(shape.cfg(), 1, 64, k)
    target_only.bind(tw)
    target_only.prefill(prompt)
    plain = Engine(shape.cfg(), 1, 64, 0)                    # prefilled token by token, without a draft step
    plain.bind(tw, dw)
    plain.prefill(prompt)
    behind = Engine(shape.cfg(), 1, 64, k)                   # two blocks committed, none drafted
    behind.bind(tw, dw)
    behind.prefill(prompt)
    none = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    for _ in range(2):
        _, ids = behind.sf_verify_step(0, none)
        behind.sf_accept_commit(0, none, ids)
    return {"target only": target_only, "plain decoding": plain, "two blocks behind": behind}


@pytest.mark.parametrize("name", SHAPES)
def test_a_prefix_without_draft_keys(name):
    """Nothing drafts from keys that were never written: the draft step is refused, the target's steps run, tails are
    prefilled."""
    k, seed, B = 2, 9, 2
    shape, tw, dw = weights(name, k, seed)
    draft = torch.ones(B, k, dtype=torch.int32, device="cuda")
    for what, one in prefixes_without_draft_keys(shape, tw, dw, k, seed).items():
        eng, ref = Engine(shape.cfg(), B, 64, k), Engine(shape.cfg(), B, 64, k)
        eng.bind(tw, dw)
        ref.bind(tw)
        for e in (eng, ref):
            e.sf_set_prefix(one)
        with pytest.raises(sfb.SfError) as e:
            eng.sf_draft_step(k)
        assert e.value.status == sfb.SF_ESTATE, what
        a, b = (x.sf_verify_step(k, draft)[0] for x in (eng, ref))
        assert torch.equal(a, b), what
        for block in (None, 8):
            tails = synth.prompts([11, 4], shape.vocab, seed + 1)
            assert torch.equal(eng.prefill(tails, block=block), ref.prefill(tails, block=block)), what
            a, b = (x.sf_verify_step(k, draft)[0] for x in (eng, ref))
            assert torch.equal(a, b), what


@pytest.mark.parametrize("block", [None, 8])
def test_sequences_without_a_tail(block):
    """A sequence whose tail is empty goes on right behind the prefix, as one that was not prefilled at all."""
    k, seed, B = 3, 11, 3
    shape, tw, dw = weights("8b-slice", k, seed)
    one, eng, ref = Engine(shape.cfg(), 1, 64, k), Engine(shape.cfg(), B, 64, k), Engine(shape.cfg(), B, 64, k)
    for e in (one, eng, ref):
        e.bind(tw, dw)
    one.prefill(synth.prompts([33], shape.vocab, seed))
    for e in (eng, ref):
        e.sf_set_prefix(one)
    tails = synth.prompts([9, 20], shape.vocab, seed + 1)
    first = eng.prefill([tails[0], tails[0][:0], tails[1]], block=block)
    assert eng.kv_len.tolist() == [9, 0, 20] and eng.n_new[1] == 1 and first[1] == one.pending[0] == eng.pending[1]
    assert torch.equal(eng.hooks[1, 0], ref.hooks[1, 0])
    a, b = (logits_of_a_draft(e, k)[1] for e in (eng, ref))
    assert torch.equal(a, b)
    draft = torch.ones(B, k, dtype=torch.int32, device="cuda")
    a, b = (e.sf_verify_step(k, draft)[0][1] for e in (eng, ref))
    assert torch.equal(a, b)
    eng.prefill([tails[0][:0]] * B, block=block)             # all of them
    assert eng.kv_len.tolist() == [0] * B and eng.pending.tolist() == one.pending.tolist() * B


def test_the_steps_workspace_outlives_the_prefix():
    """Steps may still run, on a stream of their own, when the prefix is taken away: their workspace is not given to others."""
    k, seed, B = 3, 13, 4
    shape, tw, dw = weights("8b-slice", k, seed)
    one, eng = Engine(shape.cfg(), 1, 2048, k), Engine(shape.cfg(), B, 64, k)
    for e in (one, eng):
        e.bind(tw, dw)
    one.prefill(synth.prompts([1500], shape.vocab, seed), block=64)
    eng.sf_set_prefix(one)
    n = eng.lib.sf_prefix_workspace_bytes(eng.ctx, B, k, 64) + 256
    draft = torch.ones(B, k, dtype=torch.int32, device="cuda")
    want = eng.sf_verify_step(k, draft)[0].clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = torch.empty_like(want)
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        eng.sf_verify_step(k, draft, logits_out=got)
        eng.sf_verify_step(k, draft, logits_out=got)
    eng.sf_set_prefix(None)
    others = [torch.full((n,), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(64)]
    for _ in range(200):
        for x in others:
            x.fill_(0x7f)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
