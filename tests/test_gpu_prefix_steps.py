"""Steps over a shared prefix, and sampled decoding of several continuations of one prompt as a program runs it: against the
oracle, whose sequences each hold the whole prompt."""
import numpy as np
import pytest
import torch

import sampling_oracle as so
import synth
from paper_2511_20340_amd import binding as sfb
from paper_2511_20340_amd.engine import Engine

from gpu_common import make_pair, rel_err, to_np
from test_gpu_e2e import SLICES

pytestmark = pytest.mark.gpu
SHAPES = {"tiny": (synth.TINY, 0.02), **{n: (s, 0.05) for n, s in SLICES.items()}}


def engines(shape, std, B, cap, k, seed, prompt, block=None):
    """(oracle with B copies of the prompt, engine of B sequences behind the shared prompt, the prompt's engine)"""
    orc, eng, tw, dw = make_pair(shape, B, cap, k, seed, std=std)
    one = Engine(shape.cfg(), 1, -(-(len(prompt) + k + 1) // 32) * 32, k)
    one.bind(tw, dw)
    one.prefill([prompt], block=block)
    eng.sf_set_prefix(one)
    return orc, eng, one


def commit(orc, eng, k, draft, lg_o, force, V):
    """Both commit force[b] rows of the verified block: the drafted tokens, then the oracle's choice."""
    B = orc.B
    chosen = lg_o.reshape(B, k + 1, V).argmax(-1).astype(np.int32)
    d = draft.copy()
    for b in range(B):
        chosen[b, :force[b] - 1] = draft[b, :force[b] - 1]
        if force[b] <= k:
            d[b, force[b] - 1] = (chosen[b, force[b] - 1] + 1) % V     # the next slot does not match
    planted = np.full((B, k + 1, V), -1.0, np.float32)
    np.put_along_axis(planted, chosen[..., None], 1.0, -1)
    acc_o, _ = orc.accept_commit(k, d, planted)
    acc_g, _ = eng.sf_accept_commit(k, torch.from_numpy(d).cuda(), torch.from_numpy(chosen).cuda())
    np.testing.assert_array_equal(acc_g.cpu().numpy(), acc_o)


def test_fp32_steps_follow_the_oracle():
    """Draft and verify logits of six steps that run freely; each sequence accepts another number of tokens."""
    shape, std = SHAPES["tiny"]
    B, k, seed, P = 3, 4, 41, 45
    prompt = synth.prompts([P], shape.vocab, seed)[0]
    orc, eng, one = engines(shape, std, B, 128, k, seed, prompt)
    orc.prefill([prompt] * B)
    assert int(one.pending[0]) == orc.pending[0]
    rng = np.random.default_rng(seed)
    for step in range(6):
        dl_o = orc.draft_step(k, sfb.SF_MASK_BIDIR, want_logits=True)[1]
        dl_g = torch.empty(B, k, shape.vocab, device="cuda")
        eng.sf_draft_step(k, logits_out=dl_g)
        assert rel_err(to_np(dl_g).reshape(dl_o.shape), dl_o) < 1e-4, step
        draft = rng.integers(0, shape.vocab, size=(B, k)).astype(np.int32)
        lg_o = orc.verify_step(k, draft)
        lg_g, _ = eng.sf_verify_step(k, torch.from_numpy(draft).cuda())
        assert rel_err(to_np(lg_g).reshape(lg_o.shape), lg_o) < 1e-4, step
        commit(orc, eng, k, draft, lg_o, np.array([1, k + 1, 2 + step % 2], np.int32), shape.vocab)
        np.testing.assert_array_equal(eng.kv_len.cpu().numpy() + P, orc.kv_len)


def load(orc, eng, one, P, k):
    """The oracle's state into the engines: positions below P into the prefix, the rest into the sequences' own caches."""
    L = eng.L
    for which, tables in (("tk", orc.tk), ("tv", orc.tv), ("dk", [orc.dk]), ("dv", [orc.dv])):
        for l in range(len(tables) if which[0] == "d" else L):
            t = np.asarray(tables[l])
            pre = np.zeros((1, t.shape[1], one.cap, t.shape[3]), np.float32)
            pre[0, :, :P] = t[0, :, :P]
            own = np.zeros((eng.B, t.shape[1], eng.cap, t.shape[3]), np.float32)
            own[:, :, :t.shape[2] - P] = t[:, :, P:]
            one.sf_kv_import(pre, which, l)
            eng.sf_kv_import(own, which, l)
    nn = np.minimum(orc.n_new, k + 1)
    hooks = np.zeros((eng.B, k + 1, 4, orc.d), np.float32)
    for b in range(eng.B):
        hooks[b, :nn[b]] = orc.hooks[b, orc.n_new[b] - nn[b]:orc.n_new[b]]
    eng.hooks.copy_(torch.from_numpy(hooks).cuda().to(eng.tdtype))
    eng.set_state(kv_len=orc.kv_len - P, pending=orc.pending, n_new=nn)


@pytest.mark.parametrize("name", list(SLICES))
def test_bf16_steps_teacher_forced(name):
    """Draft and verify logits, hooks and appended keys of four steps, each from the oracle's state."""
    shape, std = SHAPES[name]
    B, k, seed, P = 3, 4, 77, 40
    prompt = synth.prompts([P], shape.vocab, seed)[0]
    orc, eng, tw, dw = make_pair(shape, B, 128, k, seed, std=std, round_bf16=True)
    ref = make_pair(shape, B, 128, k, seed, std=std, round_bf16=False)[0]
    one = Engine(shape.cfg(), 1, 64, k)
    one.bind(tw, dw)
    one.prefill([prompt])
    eng.sf_set_prefix(one)
    orc.prefill([prompt] * B)
    rng = np.random.default_rng(seed)
    for step in range(4):
        ref.restore(orc.snapshot())
        if step > 0:
            load(orc, eng, one, P, k)
        orc.draft_step(k, sfb.SF_MASK_BIDIR, want_logits=True)
        dl_ref = ref.draft_step(k, sfb.SF_MASK_BIDIR, want_logits=True)[1]
        if step == 0:
            load(orc, eng, one, P, k)              # the oracle's draft cache holds the prompt only now
        dl_g = torch.empty(B, k, shape.vocab, device="cuda")
        eng.sf_draft_step(k, logits_out=dl_g)
        assert rel_err(to_np(dl_g).reshape(dl_ref.shape), dl_ref) < 2e-2, step
        draft = rng.integers(0, shape.vocab, size=(B, k)).astype(np.int32)
        lg_o = orc.verify_step(k, draft)
        lg_g, ids = eng.sf_verify_step(k, torch.from_numpy(draft).cuda())
        assert rel_err(to_np(lg_g).reshape(lg_o.shape), lg_o) < 2e-2, step
        assert torch.equal(ids.long(), lg_g.argmax(-1))
        assert rel_err(to_np(eng.hooks), orc.hooks[:, :k + 1]) < 2e-2
        for l in (0, shape.n_layers - 1):
            got = to_np(eng.sf_kv_export("tk", l))
            for b in range(B):
                n = int(orc.kv_len[b]) + k + 1
                assert rel_err(got[b, :, :n - P], orc.tk[l][b, :, P:n]) < 2e-2
        commit(orc, eng, k, draft, lg_o, np.array([1, k + 1, 2 + step % 2], np.int32), shape.vocab)


@pytest.mark.parametrize("name", ["tiny", "8b-slice"])
def test_tails_behind_the_prefix_are_prefilled(name):
    """Every sequence adds a tail of its own to the shared prompt, in blocks of several lengths.  fp32: a step then follows the
    oracle.  bf16: the first layer's keys and values, which hang on tokens and positions alone, are those of an engine that
    holds the whole prompts, bit for bit."""
    shape, std = SHAPES[name]
    B, k, seed, P = 3, 3, 43, 40
    prompt = synth.prompts([P], shape.vocab, seed)[0]
    tails = synth.prompts([5, 21, 12], shape.vocab, seed + 1)
    whole = [np.concatenate([prompt, t]) for t in tails]
    for block in (None, 8):
        orc, eng, one = engines(shape, std, B, 96, k, seed, prompt)
        eng.prefill(tails, block=block)
        lens = eng.kv_len.cpu().numpy()
        np.testing.assert_array_equal(lens, [len(t) for t in tails])
        if shape.dtype == "bf16":
            plain = make_pair(shape, B, 96, k, seed, std=std)[1]
            plain.prefill(whole)
            for which in ("tk", "tv"):
                a, b = eng.sf_kv_export(which, 0), plain.sf_kv_export(which, 0)
                for i in range(B):
                    assert torch.equal(a[i, :, :lens[i]], b[i, :, P:P + lens[i]]), (which, i, block)
            continue
        orc.prefill(whole)
        eng.pending.copy_(torch.from_numpy(orc.pending.astype(np.int32)))
        dl_o = orc.draft_step(k, sfb.SF_MASK_BIDIR, want_logits=True)[1]
        dl_g = torch.empty(B, k, shape.vocab, device="cuda")
        eng.sf_draft_step(k, logits_out=dl_g)
        assert rel_err(to_np(dl_g).reshape(dl_o.shape), dl_o) < 1e-4
        draft = np.ones((B, k), np.int32)
        lg_o = orc.verify_step(k, draft)
        lg_g, _ = eng.sf_verify_step(k, torch.from_numpy(draft).cuda())
        assert rel_err(to_np(lg_g).reshape(lg_o.shape), lg_o) < 1e-4


@pytest.mark.parametrize("greedy_draft", [False, True])
def test_sampled_decoding_of_one_prompt(greedy_draft):
    """draft -> draw -> verify -> accept and commit at temperature > 0, the sequences of a batch behind one prompt: every
    decision is the definition's on the engine's own logits, and the loop runs on."""
    shape, std = SHAPES["8b-slice"]
    B, k, seed = 6, 3, 47
    prompt = synth.prompts([50], shape.vocab, seed)[0]
    _, eng, one = engines(shape, std, B, 96, k, seed, prompt)
    V = shape.vocab
    per = [(0.8, 0, 0.9, 0.0), (1.0, 20, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.2, 50, 0.95, 0.02), (1.0, 0, 1.0, 0.0), (0.7, 0, 1.0, 0.1)]
    t, tk, tp, mp = zip(*per)
    s = (torch.tensor(t, device="cuda"), torch.tensor(tk, dtype=torch.int32, device="cuda"), torch.tensor(tp, device="cuda"),
         torch.tensor(mp, device="cuda"))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dl, seen = torch.empty(B, k, V, device="cuda"), []
    for step in range(6):
        kv0 = eng.kv_len.clone()
        draft = eng.sf_draft_step(k, logits_out=dl)
        more = {}
        if not greedy_draft:
            ud = torch.rand(B * k, generator=g, device="cuda")
            draft, dist = eng.sf_op_sample(dl.view(B * k, V), ud, *s, group=k, want_dist=True)
            draft = draft.view(B, k)
            more = dict(draft_logits=dl, draft_dist=dist)
        logits, _ = eng.sf_verify_step(k, draft)
        ua, us = torch.rand(B, k, generator=g, device="cuda"), torch.rand(B, generator=g, device="cuda")
        acc, out = eng.sf_accept_commit_sampled(k, draft, logits, ua, us, *s, **more)
        for b in range(B):
            qw = None if greedy_draft else [so.kept_weights(dl[b, i].cpu().numpy(), *per[b]) for i in range(k)]
            n, token, w = so.accept(draft[b].cpu().numpy(), logits[b].cpu().numpy(), ua[b].cpu().numpy(), float(us[b]), per[b], qw)
            assert int(acc[b]) == n + 1, (step, b)
            got = int(out[b, n])
            assert got == token or so.near_border(w, float(us[b]), got), (step, b)
        assert torch.equal(eng.kv_len, kv0 + acc) and torch.equal(eng.pending, out.gather(1, (acc - 1).long()[:, None])[:, 0])
        seen.append(out[:, 0].cpu().numpy())
    assert eng.sf_check_state() == 0
    with pytest.raises(sfb.SfError) as e:                            # one block is committed once
        eng.sf_accept_commit_sampled(k, draft, logits, ua, us, *s, **more)
    assert e.value.status == sfb.SF_ESTATE
    assert len({tuple(x) for x in np.array(seen).T}) > 1             # the continuations differ


def test_a_captured_step_over_the_prefix():
    """The sampled step in a HIP graph, replayed: the eager bits."""
    shape, std = SHAPES["8b-slice"]
    B, k, seed, V = 4, 2, 53, SHAPES["8b-slice"][0].vocab
    prompt = synth.prompts([70], shape.vocab, seed)[0]
    _, a, one = engines(shape, std, B, 96, k, seed, prompt)
    _, b, one_b = engines(shape, std, B, 96, k, seed, prompt)
    ud, ua, us = (torch.empty(n, device="cuda") for n in ((B * k,), (B, k), (B,)))
    dl, lg = torch.empty(B, k, V, device="cuda"), torch.empty(B, k + 1, V, device="cuda")
    ids = torch.empty(B, k + 1, dtype=torch.int32, device="cuda")
    t = torch.full((B,), 0.9, device="cuda")

    def step(e):
        greedy = e.sf_draft_step(k, logits_out=dl)
        draft, dist = e.sf_op_sample(dl.view(B * k, V), ud, t, group=k, want_dist=True)
        draft = draft.view(B, k)
        e.sf_verify_step(k, draft, logits_out=lg, ids_out=ids)
        return e.sf_accept_commit_sampled(k, draft, lg, ua, us, t, draft_logits=dl, draft_dist=dist)
    keep = {n: getattr(a, n).clone() for n in ("kv_len", "pending", "n_new", "cu_new", "hooks")}
    for e in (a, b):
        e.pin_len_upper()
    for u in (ud, ua, us):
        u.uniform_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a)
    for n, x in keep.items():
        getattr(a, n).copy_(x)
    for it in range(5):
        for u in (ud, ua, us):
            u.uniform_()
        want = [x.clone() for x in step(b)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), it
        for n in keep:
            assert torch.equal(getattr(a, n), getattr(b, n)), (it, n)


def test_set_prefix_refuses_and_ends():
    shape, std = SHAPES["tiny"]
    prompt = synth.prompts([20], shape.vocab, 3)[0]
    _, eng, one = engines(shape, std, 2, 64, 2, 3, prompt)
    with pytest.raises(sfb.SfError) as e:
        eng.sf_draft_step(2, mask=sfb.SF_MASK_BIDIR | sfb.SF_DRAFT_TWO_STAGE)
    assert e.value.status in (sfb.SF_EUNSUPPORTED, sfb.SF_ESTATE)
    for bad in (dict(length=21), dict(length=0), dict(length=5)):
        with pytest.raises(ValueError):
            eng.sf_set_prefix(one, **bad)
    with pytest.raises(ValueError):
        eng.sf_set_prefix(eng)
    eng.sf_set_prefix(None)
    _, ref, _, _ = make_pair(shape, 2, 64, 2, 3)
    prompts = synth.prompts([9, 14], shape.vocab, 4)
    assert torch.equal(eng.prefill(prompts), ref.prefill(prompts))
    a, b = (x.sf_verify_step(2, torch.ones(2, 2, dtype=torch.int32, device="cuda"))[0] for x in (eng, ref))
    assert torch.equal(a, b)


def test_a_refused_prefix_leaves_the_one_before():
    """What is refused changes nothing; an engine's own caches and a prefix behind a prefix are; a pinned bound stays pinned."""
    shape, std = SHAPES["tiny"]
    _, eng, one = engines(shape, std, 1, 64, 2, 5, synth.prompts([20], shape.vocab, 5)[0])
    kept, draft = eng._prefix, torch.ones(1, 2, dtype=torch.int32, device="cuda")
    want = eng.sf_verify_step(2, draft)[0].clone()
    third = Engine(shape.cfg(), 1, 64, 2)
    for bad in (eng, Engine(shape.cfg(), 1, 64, 2, share_caches=eng)):
        with pytest.raises(ValueError):
            eng.sf_set_prefix(bad, start=False)
    with pytest.raises(ValueError):
        third.sf_set_prefix(eng)
    with pytest.raises(ValueError):
        eng.sf_set_prefix(one, length=21)
    assert eng._prefix is kept and torch.equal(eng.sf_verify_step(2, draft)[0], want)
    eng.pin_len_upper()
    bound = eng.len_upper
    eng.sf_set_prefix(one)
    assert eng.len_upper == bound and torch.equal(eng.sf_verify_step(2, draft)[0], want)
    assert eng.sf_check_state() == 0
