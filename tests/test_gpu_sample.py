"""sf_op_sample and sf_op_accept_sampled against their definition in doubles (tests/sampling_oracle.py): sizes, settings and
rows where a selection can go wrong, acceptance in distribution, capture, streams, wide offsets."""
import numpy as np
import pytest
import torch

import sampling_oracle as so
from paper_2511_20340_amd.engine import Engine

pytestmark = pytest.mark.gpu

OFF = (1.0, 0, 1.0, 0.0)


def engine(B=1, k=1, vocab=64):
    return Engine({"n_layers": 1, "d_model": 64, "n_q_heads": 1, "n_kv_heads": 1, "head_dim": 64, "d_ffn": 64, "vocab": vocab,
                   "dtype": "bf16"}, B, 32, k)


@pytest.fixture(scope="module")
def eng():
    return engine()


def cuda(a, dtype=torch.float32):
    return torch.as_tensor(np.asarray(a)).to(dtype).cuda().contiguous()


def settings_of(per_row):
    t, k, p, m = zip(*per_row)
    return cuda(t), cuda(k, torch.int32), cuda(p), cuda(m)


def check(eng, rows, per_row, u):
    """Every row of `rows` with its settings and number: token and probability as the definition has them."""
    rows = np.asarray(rows, np.float32)
    ids, prob = eng.sf_op_sample(cuda(rows), cuda(u), *settings_of(per_row), want_prob=True)
    ids, prob = ids.cpu().numpy(), prob.cpu().numpy()
    for r in range(len(rows)):
        w = so.kept_weights(rows[r], *per_row[r])
        if not w.sum() > 0:
            assert ids[r] == 0 and prob[r] == 0
            continue
        assert so.near_border(w, u[r], ids[r]), (r, per_row[r], u[r], ids[r], so.draw(w, u[r]))
        want = w[ids[r]] / w.sum()
        # the share is a double of relative error (n + 8) 2^-53, rounded once to float
        assert abs(prob[r] - want) <= want * (2.0 ** -24 + (len(w) + 8) * 2.0 ** -53) + 2.0 ** -150, (r, per_row[r])


MIX = [OFF, (0.7, 0, 1.0, 0.0), (1.0, 5, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.8, 50, 0.95, 0.05), (1.3, 0, 0.5, 0.0),
       (1.0, 0, 1.0, 0.1), (0.0, 7, 0.9, 0.2), (1.0, 1, 0.3, 0.0), (2.0, 1000, 0.99, 0.0), (1.0, 0, 0.0, 0.0),
       (1.0, 3, 1e-9, 0.0), (0.6, 200, 0.98, 1.0), (1.0, 0, 0.9999, 1e-6)]


@pytest.mark.parametrize("V", [1, 2, 3, 5, 63, 64, 65, 255, 256, 257, 1000, 1024, 4097, 8191, 8193, 32003, 70001, 131072])
def test_sizes_and_settings(eng, V):
    rng = np.random.default_rng(V)
    rows = rng.normal(size=(2 * len(MIX), V)).astype(np.float32) * 2
    rows[::2] += 9 * (rng.random(rows[::2].shape) < 20 / V)
    check(eng, rows, MIX + MIX, rng.random(len(rows)).astype(np.float32))


def odd_rows(V, rng):
    """Rows of values that a selection meets at its limits."""
    g = rng.normal(size=V).astype(np.float32)
    half, few = rng.random(V) < 0.5, rng.random(V) < 0.01
    yield "equal", np.full(V, 1.5, np.float32)
    yield "two values", np.where(half, 1.0, -1.0)
    yield "three values, the best rare", np.where(few, 2.0, np.where(half, 1.0, 0.5))
    yield "coarse grid", np.round(g * 2) / 2
    yield "zeros of both signs", np.where(half, 0.0, -0.0)
    yield "half masked", np.where(half, -np.inf, g)
    yield "nearly all masked", np.where(few, g, -np.inf)
    yield "masked by the lowest value", np.where(half, np.finfo(np.float32).min, g)
    yield "NaN among them", np.where(half, np.nan, g)
    yield "NaN and masks", np.where(few, np.nan, np.where(half, -np.inf, g))
    yield "infinite", np.where(few, np.inf, g)
    yield "infinite and masked", np.where(few, np.inf, -np.inf)
    yield "all masked", np.full(V, -np.inf)
    yield "all NaN", np.full(V, np.nan)
    yield "NaN first, then masks", np.concatenate([[np.nan], np.full(V - 1, -np.inf)])
    yield "largest and lowest values", np.where(half, np.finfo(np.float32).max, np.finfo(np.float32).min)
    yield "tiny values", (g * 1e-40).astype(np.float32)
    yield "all scales", np.sign(g) * 10.0 ** rng.uniform(-44, 38, V)
    yield "far apart", g * 1e4
    yield "one token", np.where(np.arange(V) == V // 2, 3.0, -np.inf)
    yield "a flat crowd under one", np.where(np.arange(V) == V - 1, 8.0, 0.0)
    yield "close together", 1.0 + np.arange(V) % 7 * 2.0 ** -23


@pytest.mark.parametrize("V", [4, 300, 5000, 20011])
def test_rows_at_the_limits(eng, V):
    rng = np.random.default_rng(V + 1)
    with np.errstate(over="ignore"):
        rows = [(n, np.asarray(x).astype(np.float32)) for n, x in odd_rows(V, rng)]
    for name, x in rows:
        print(name, flush=True)
        u = rng.random(len(MIX)).astype(np.float32)
        u[:4] = 0.0, 1 - 2.0 ** -24, 0.5, 0.25
        check(eng, np.tile(x, (len(MIX), 1)), MIX, u)


def test_temperatures_at_the_limits(eng):
    rng = np.random.default_rng(3)
    x = rng.normal(size=4000).astype(np.float32)
    x[::5] = -np.inf
    ts = [1e-45, 1e-30, 1e-3, 50.0, 1e30, 3e38, np.inf, -1.0, np.nan]
    per = [(t, k, p, 0.0) for t in ts for k, p in ((0, 1.0), (17, 1.0), (0, 0.9), (3000, 0.7))]
    check(eng, np.tile(x, (len(per), 1)), per, rng.random(len(per)).astype(np.float32))


@pytest.mark.parametrize("V", [700, 12095, 33000, 131072])
def test_large_counts(eng, V):
    """Counts around what is ranked one by one, what LDS has room for and what a row has unmasked."""
    rng = np.random.default_rng(V + 2)
    x = (rng.normal(size=(4, V)) * 1.8).astype(np.float32)
    x[1, rng.random(V) < 0.9] = -np.inf
    x[2] = np.round(x[2] * 8) / 8
    x[3, rng.random(V) < 0.995] = -np.inf
    per = [(t, k, p, m) for k in (300, 512, 1000, 1535, 1537, 4096, 4097, 8200, 20000)
           for t, p, m in ((1.0, 1.0, 0.0), (0.7, 0.9, 0.0), (3.0, 0.98, 0.0), (1.3, 0.95, 0.05))]
    for row in x:
        check(eng, np.tile(row, (len(per), 1)), per, rng.random(len(per)).astype(np.float32))


def test_numbers_outside_the_unit_interval(eng):
    x = np.random.default_rng(4).normal(size=1000).astype(np.float32)
    x[990:] = -np.inf
    u = np.array([0.0, -0.5, 1.0, 7.0, np.nan, np.inf, -np.inf], np.float32)
    ids = eng.sf_op_sample(cuda(np.tile(x, (7, 1))), cuda(u)).cpu().numpy()
    assert list(ids) == [0, 0, 989, 989, 989, 989, 0]


def test_settings_by_group_and_absent_ones(eng):
    rng = np.random.default_rng(5)
    rows, u = rng.normal(size=(7, 999)).astype(np.float32), rng.random(7).astype(np.float32)
    t, k, p, m = settings_of([(0.5, 0, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 4, 1.0, 0.0)])
    whole = eng.sf_op_sample(cuda(rows), cuda(u), t, k, p, m, group=3)
    each = eng.sf_op_sample(cuda(rows), cuda(u), *(s.repeat_interleave(3)[:7].contiguous() for s in (t, k, p, m)))
    assert torch.equal(whole, each)
    assert torch.equal(eng.sf_op_sample(cuda(rows), cuda(u)), eng.sf_op_sample(cuda(rows), cuda(u), *settings_of([OFF] * 7)))
    assert torch.equal(eng.sf_op_sample(cuda(rows), cuda(u), temperature=torch.zeros(7, device="cuda")),
                       eng.sf_op_argmax(cuda(rows)))


def test_rows_off_16_bytes_and_behind_4_gib(eng):
    rng = np.random.default_rng(6)
    V, M = 131071, 16500                                    # 2.16e9 logits
    big = torch.zeros(M * V + 3, device="cuda")
    for off in (1, 3):
        x = big[off:off + M * V].view(M, V)
        row = rng.normal(size=V).astype(np.float32) * 2
        x[-1] = cuda(row)
        u = torch.full((M,), 0.37, device="cuda")
        k = torch.zeros(M, dtype=torch.int32, device="cuda")
        k[-1] = 40
        ids = eng.sf_op_sample(x, u, top_k=k)
        assert so.near_border(so.kept_weights(row, 1.0, 40), 0.37, int(ids[-1]))
        # equal logits: the running weights are whole numbers
        assert (ids[:-1] == int(np.floor(float(np.float32(0.37)) * V))).all()
        x[-1] = 0


def accept_case(B, k, V, seed, sampled, per, eng):
    rng = np.random.default_rng(seed)
    target = rng.normal(size=(B, k + 1, V)).astype(np.float32) * 2
    dl = target[:, :k] + rng.normal(size=(B, k, V)).astype(np.float32)
    ua, us, ud = (rng.random(s).astype(np.float32) for s in ((B, k), (B,), (B, k)))
    qw = None
    if sampled:
        qw = np.array([[so.kept_weights(dl[b, i], *per[b]) for i in range(k)] for b in range(B)])
        draft = np.array([[so.draw(qw[b, i], ud[b, i]) for i in range(k)] for b in range(B)], np.int32).reshape(B, k)
    else:
        draft = dl.argmax(-1).astype(np.int32) if k else np.zeros((B, 0), np.int32)
    return target, dl, draft, ua, us, ud, qw


def run_accept(eng, k, target, dl, draft, ua, us, ud, per, sampled):
    B, V = target.shape[0], target.shape[2]
    s = settings_of(per)
    more = {}
    if sampled and k:
        d = cuda(dl)
        _, dist = eng.sf_op_sample(d.view(B * k, V), cuda(ud).view(-1), *s, group=k, want_dist=True)
        more = dict(draft_logits=d, draft_dist=dist)
    return eng.sf_op_accept_sampled(k, cuda(draft, torch.int32), cuda(target), cuda(ua), cuda(us), *s, **more)


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("B,k,V", [(1, 0, 5), (1, 1, 1), (3, 4, 2), (14, 4, 777), (14, 7, 8193), (28, 2, 20001), (1, 127, 64), (14, 3, 70001)])
def test_acceptance(B, k, V, sampled):
    eng = engine(B, max(k, 1))
    per = [MIX[b % len(MIX)] for b in range(B)]
    target, dl, draft, ua, us, ud, qw = accept_case(B, k, V, B * 100 + k, sampled and k > 0, per, eng)
    kv0 = np.arange(B, dtype=np.int32) * 3
    eng.kv_len.copy_(torch.from_numpy(kv0))
    acc, out = run_accept(eng, k, target, dl, draft, ua, us, ud, per, sampled)
    acc, out = acc.cpu().numpy(), out.cpu().numpy()
    for b in range(B):
        n, token, w = so.accept(draft[b], target[b], ua[b], us[b], per[b], qw[b] if qw is not None else None)
        assert acc[b] == n + 1, (b, per[b])
        assert list(out[b, :n]) == list(draft[b, :n]) and (out[b, n + 1:] == -1).all()
        assert out[b, n] == token or so.near_border(w, us[b], out[b, n]), (b, per[b])
    a = acc.astype(np.int64)
    np.testing.assert_array_equal(eng.kv_len.cpu().numpy(), kv0 + a)
    np.testing.assert_array_equal(eng.n_new.cpu().numpy(), a)
    np.testing.assert_array_equal(eng.cu_new.cpu().numpy(), np.concatenate([[0], np.cumsum(a)]))
    np.testing.assert_array_equal(eng.pending.cpu().numpy(), out[np.arange(B), a - 1])


def test_acceptance_of_strange_drafts():
    """Ids outside the vocabulary, tokens that the target masks, a draft that equals the target, rows without a token."""
    V, k, B = 300, 2, 6
    eng = engine(B, k)
    rng = np.random.default_rng(8)
    target = rng.normal(size=(B, k + 1, V)).astype(np.float32)
    draft = rng.integers(0, V, size=(B, k)).astype(np.int32)
    draft[0] = -1, 5
    draft[1] = V, 5
    target[2, 0, draft[2, 0]] = -np.inf
    target[4, 0] = -np.inf
    target[5, 0] = np.nan
    dl = target[:, :k].copy()
    dl[3, 0, :] = target[3, 0]
    draft[3, 0] = -7                                       # same distribution, and the drafted token has no share in it
    per, u = [OFF] * B, rng.random
    ua, us, ud = u((B, k)).astype(np.float32), u(B).astype(np.float32), u((B, k)).astype(np.float32)
    for sampled in (True, False):
        qw = np.array([[so.kept_weights(dl[b, i]) for i in range(k)] for b in range(B)]) if sampled else None
        acc, out = run_accept(eng, k, target, dl, draft, ua, us, ud, per, sampled)
        acc, out = acc.cpu().numpy(), out.cpu().numpy()
        for b in range(B):
            n, token, w = so.accept(draft[b], target[b], ua[b], us[b], per[b], qw[b] if sampled else None)
            assert acc[b] == n + 1 and (out[b, n] == token or so.near_border(w, us[b], out[b, n])), (sampled, b)
            assert (out[b, :acc[b]] >= 0).all() and (out[b, :acc[b]] < V).all()


def test_greedy_acceptance_is_the_greedy_rule():
    B, k, V = 9, 4, 500
    a, b = engine(B, k), engine(B, k)
    rng = np.random.default_rng(9)
    target = cuda(rng.normal(size=(B, k + 1, V)))
    ids = a.sf_op_argmax(target.view(-1, V)).view(B, k + 1)
    draft = ids[:, :k].clone()
    draft[torch.rand(B, k, device="cuda") < 0.3] += 1
    draft = (draft % V).contiguous()
    zero = torch.zeros(B, device="cuda")
    want = a.sf_op_accept(k, draft, ids)
    got = b.sf_op_accept_sampled(k, draft, target, torch.rand(B, k, device="cuda"), torch.rand(B, device="cuda"), temperature=zero)
    for x, y in zip(want, got):
        assert torch.equal(x, y)
    for n in ("kv_len", "pending", "n_new", "cu_new"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n


@pytest.mark.parametrize("sampled", [True, False])
def test_acceptance_keeps_the_targets_distribution(sampled):
    """Whatever the draft proposes, the first token of a block follows the target's distribution: 4096 blocks, frequencies
    within six standard deviations, sqrt(p (1 - p) / n) each."""
    B, k, V = 4096, 2, 8
    eng = engine(B, k)
    rng = np.random.default_rng(10)
    per = (0.9, 6, 0.95, 0.0)
    t1, d1 = rng.normal(size=(k + 1, V)).astype(np.float32) * 1.5, rng.normal(size=(k, V)).astype(np.float32) * 1.5
    target, dl = cuda(np.tile(t1, (B, 1, 1))), cuda(np.tile(d1, (B, 1, 1)))
    s = settings_of([per] * B)
    more, ud = {}, cuda(rng.random((B * k,)))
    if sampled:
        draft, dist = eng.sf_op_sample(dl.view(B * k, V), ud, *s, group=k, want_dist=True)
        draft = draft.view(B, k)
        more = dict(draft_logits=dl, draft_dist=dist)
    else:
        draft = dl.argmax(-1).to(torch.int32)
    acc, out = eng.sf_op_accept_sampled(k, draft, target, cuda(rng.random((B, k))), cuda(rng.random(B)), *s, **more)
    p = so.kept_weights(t1[0], *per)
    p /= p.sum()
    n = np.bincount(out[:, 0].cpu().numpy(), minlength=V)
    assert (np.abs(n / B - p) <= 6 * np.sqrt(p * (1 - p) / B)).all(), (n / B, p)
    if sampled:
        q = so.kept_weights(d1[0], *per)
        rate = np.minimum(p, q / q.sum()).sum()
        assert abs(float((acc > 1).float().mean()) - rate) <= 6 * np.sqrt(rate * (1 - rate) / B)


def test_captured_and_on_another_stream():
    """A captured draw and acceptance, replayed over new inputs between eager work, has the eager bits each time."""
    B, k, V = 6, 3, 5003
    eng, ref = engine(B, k), engine(B, k)
    s = settings_of([MIX[b] for b in range(B)])
    dl, target = torch.empty(B, k, V, device="cuda"), torch.empty(B, k + 1, V, device="cuda")
    ud, ua, us = (torch.empty(n, device="cuda") for n in ((B * k,), (B, k), (B,)))

    def fill(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        target.normal_(generator=g)
        target.mul_(3)
        dl.copy_(target[:, :k] + torch.randn(B, k, V, generator=g, device="cuda"))
        for u in (ud, ua, us):
            u.uniform_(generator=g)

    def step(e):
        draft, dist = e.sf_op_sample(dl.view(B * k, V), ud, *s, group=k, want_dist=True)
        draft = draft.view(B, k)
        return (draft,) + tuple(e.sf_op_accept_sampled(k, draft, target, ua, us, *s, draft_logits=dl, draft_dist=dist))
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(eng)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(eng)
    for it in range(5):
        fill(it + 1)
        for e in (eng, ref):
            e.kv_len.fill_(it)
        want = step(ref)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), it
        for n in ("kv_len", "pending", "n_new", "cu_new"):
            assert torch.equal(getattr(eng, n), getattr(ref, n)), (it, n)
        with torch.cuda.stream(side):                       # and on a stream of its own
            side.wait_stream(torch.cuda.current_stream())
            ref.kv_len.fill_(it)
            other = step(ref)
        side.synchronize()
        for x, y in zip(other, want):
            assert torch.equal(x, y), it
