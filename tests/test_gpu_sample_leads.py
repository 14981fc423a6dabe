"""Rows whose largest logit leads a patterned crowd by more than the lists of the segments reach (32 logits): draws and
acceptance against the definition, and the rows next to them, whose lists lie behind in the workspace."""
import numpy as np
import pytest
import torch

import sampling_oracle as so
from test_gpu_sample import check, cuda, eng, engine, run_accept, settings_of  # noqa: F401

pytestmark = pytest.mark.gpu

SETTINGS = [(1.0, 50, 1.0, 0.0), (1.0, 0, 1.0, 1e-15), (0.7, 20, 0.9, 0.0), (2.0, 256, 1.0, 0.0), (1.3, 2, 1.0, 0.0), (1.0, 0, 1.0, 1e-30),
            (1.0, 256, 0.95, 1e-20), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.0)]


def patterned(V, every, low, lead):
    x = np.full(V, low, np.float32)
    x[::every] = 0.0
    x[V // 3] = lead
    return x


def allowed(V, rng, low, lead):
    """One allowed token for each four of 1024, the rest lowered by a finite mask."""
    x = np.full(V, low, np.float32)
    at = np.arange(0, min(V, 1024) - 4, 4)
    at = at + 1024 * rng.integers(0, max(1, V // 1024 - 1), len(at))
    x[at] = rng.normal(size=len(at))
    x[V // 2] = lead
    return x


@pytest.mark.parametrize("V", [8192, 32000, 8191, 700])
def test_draws(eng, V):  # noqa: F811
    rng = np.random.default_rng(V)
    for lead in (33.0, 40.0, 64.5, 100.0):
        rows = [patterned(V, e, -1.0, lead) for e in (17, 18, 26, 30)] + [patterned(V, 17, -1e4, lead)]
        rows += [allowed(V, rng, low, lead) for low in (-50.0, -1e4)] + [rng.normal(size=V).astype(np.float32)]
        for row in rows:                                    # alone
            check(eng, row[None], SETTINGS[:1], np.array([0.3], np.float32))
        per = [s for s in SETTINGS for _ in rows]
        check(eng, np.tile(np.stack(rows), (len(SETTINGS), 1)), per, rng.random(len(per)).astype(np.float32))


@pytest.mark.parametrize("sampled", [True, False])
def test_acceptance(sampled):
    B, k, V = len(SETTINGS), 3, 8192
    e = engine(B, k)
    rng = np.random.default_rng(12)
    target = np.stack([np.stack([patterned(V, 17 + b, -1.0, 40.0 if i % 2 else 34.0) for i in range(k + 1)]) for b in range(B)])
    dl = np.stack([np.stack([patterned(V, 17, -1.0, 36.0) for _ in range(k)]) for _ in range(B)])
    dl[1::2, 0, V // 3], dl[1::2, 0, 17] = -1.0, 45.0       # another leader: nothing is accepted
    ua, us, ud = (rng.random(s).astype(np.float32) for s in ((B, k), (B,), (B, k)))
    qw = np.array([[so.kept_weights(dl[b, i], *SETTINGS[b]) for i in range(k)] for b in range(B)])
    draft = np.array([[so.draw(qw[b, i], ud[b, i]) for i in range(k)] for b in range(B)], np.int32)
    if not sampled:
        draft, qw = dl.argmax(-1).astype(np.int32), None
    acc, out = run_accept(e, k, target, dl, draft, ua, us, ud, SETTINGS, sampled)
    acc, out = acc.cpu().numpy(), out.cpu().numpy()
    for b in range(B):
        n, token, w = so.accept(draft[b], target[b], ua[b], us[b], SETTINGS[b], qw[b] if sampled else None)
        assert acc[b] == n + 1, b
        assert out[b, n] == token or so.near_border(w, us[b], out[b, n]), b


def test_the_workspace_ends_where_it_says(eng):  # noqa: F811
    """Rows of that kind at the end of the workspace: what lies behind it stays as it was."""
    V, M = 8192, 3
    x = cuda(np.stack([patterned(V, e, -1.0, 40.0) for e in (17, 20, 28)]))
    u, t, k, p, m = (cuda(np.full(M, 0.4)),) + settings_of([(1.0, 50, 1.0, 0.0)] * M)
    nb = eng.lib.sf_sample_workspace_bytes(M, V)
    ws = torch.full((nb + (1 << 16),), 0x5a, dtype=torch.uint8, device="cuda")
    at = ws.data_ptr() + (-ws.data_ptr()) % 256
    ids = torch.empty(M, dtype=torch.int32, device="cuda")
    par = eng._sampling("test", M, t, k, p, m)
    assert eng.lib.sf_op_sample(eng.ctx, x.data_ptr(), M, V, 1, par, u.data_ptr(), ids.data_ptr(), None, None, at, nb,
                                torch.cuda.current_stream().cuda_stream) == 0
    assert ids.tolist() == [V // 3] * M
    assert (ws[at - ws.data_ptr() + nb:] == 0x5a).all()
