"""What a context and an engine know about a shared prefix: calls in another order."""
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
