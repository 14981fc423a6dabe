"""Refusals of the sampling entry points, on the host: status codes before anything is launched, and the engine's checks."""
import ctypes as C

import numpy as np
import pytest

import sampling_oracle as so
from paper_2511_20340_amd import binding as sfb
from test_abi import cfg, create

FAKE = 0x10000


def test_sample_validates_before_launching_anything():
    L = sfb.lib()
    st, ctx = create(cfg(), cfg(n_layers=1))
    assert st == sfb.SF_OK
    par = sfb.Sampling()

    def call(**kw):
        a = dict(ctx=ctx, x=FAKE, M=4, V=1000, group=1, u=FAKE, ids=FAKE, dist=None, ws=FAKE, nb=1 << 30)
        a.update(kw)
        return L.sf_op_sample(a["ctx"], a["x"], a["M"], a["V"], a["group"], C.byref(par), a["u"], a["ids"], None, a["dist"],
                              a["ws"], a["nb"], None)
    for bad in (dict(ctx=None), dict(x=None), dict(u=None), dict(ids=None), dict(M=0), dict(M=-1), dict(V=0), dict(group=0),
                dict(dist=FAKE + 4)):
        assert call(**bad) == sfb.SF_EINVAL, bad
    assert call(V=(1 << 20) + 1) == sfb.SF_EUNSUPPORTED
    assert call(M=(1 << 20) + 1, V=1) == sfb.SF_EUNSUPPORTED
    need = L.sf_sample_workspace_bytes(4, 1000)
    if need:
        assert call(nb=need - 1) == sfb.SF_ECAPACITY
        assert call(ws=FAKE + 16) == sfb.SF_ECAPACITY
        assert call(ws=None) == sfb.SF_ECAPACITY
    assert L.sf_sample_workspace_bytes(0, 10) == 0 and L.sf_sample_workspace_bytes(10, 0) == 0
    assert L.sf_sample_dist_bytes(0) == 0 and L.sf_sample_dist_bytes(3) == 3 * L.sf_sample_dist_bytes(1) > 0
    assert L.sf_last_hip_error(ctx) == 0
    L.sf_destroy(ctx)


def test_accept_sampled_validates_before_launching_anything():
    L = sfb.lib()
    st, ctx = create(cfg(), cfg(n_layers=1))
    assert st == sfb.SF_OK
    need = L.sf_accept_sampled_workspace_bytes(4, 3, 1000)
    assert need > 0
    for bad in ((0, 3, 1000), (4, -1, 1000), (4, 128, 1000), (4, 3, 0)):
        assert L.sf_accept_sampled_workspace_bytes(*bad) == 0

    def call(**kw):
        a = dict(ctx=ctx, B=4, k=3, V=1000, draft=FAKE, target=FAKE, dl=FAKE, dd=FAKE, ua=FAKE, us=FAKE, acc=FAKE, out=FAKE, kv=FAKE,
                 pending=FAKE, n_new=FAKE, cu=FAKE, ws=FAKE, nb=need)
        a.update(kw)
        return L.sf_op_accept_sampled(a["ctx"], a["B"], a["k"], a["V"], a["draft"], a["target"], None, a["dl"], a["dd"], a["ua"],
                                      a["us"], a["acc"], a["out"], a["kv"], a["pending"], a["n_new"], a["cu"], a["ws"], a["nb"], None)
    for bad in (dict(ctx=None), dict(B=0), dict(k=-1), dict(k=128), dict(V=0), dict(draft=None), dict(target=None), dict(dd=None),
                dict(dd=FAKE + 4), dict(ua=None), dict(us=None), dict(acc=None), dict(out=None), dict(kv=None), dict(pending=None),
                dict(n_new=None), dict(cu=None), dict(ws=None), dict(ws=FAKE + 8)):
        assert call(**bad) == sfb.SF_EINVAL, bad
    assert call(nb=need - 1) == sfb.SF_ECAPACITY
    assert call(V=(1 << 20) + 1) == sfb.SF_EUNSUPPORTED
    assert call(B=1 << 20) == sfb.SF_EUNSUPPORTED
    # on a state: bound, and a verified block to commit
    s = sfb.State()
    commit = lambda: L.sf_accept_commit_sampled(ctx, C.byref(s), 3, FAKE, FAKE, None, None, None, FAKE, FAKE, FAKE, FAKE, FAKE,  # noqa: E731
                                                1 << 30, None)
    assert commit() == sfb.SF_ESTATE
    tw = sfb.TargetWeights()
    arr = (C.c_void_p * 2)(FAKE, FAKE)
    for n, _ in sfb.TargetWeights._fields_:
        setattr(tw, n, arr if n not in ("embed", "lm_head", "final_norm") else FAKE)
    assert L.sf_bind(ctx, C.byref(tw), None) == sfb.SF_OK
    for n in ("tk", "tv", "dk", "dv", "kv_len", "pending", "hooks", "n_new", "cu_new"):
        setattr(s, n, FAKE)
    s.B, s.cap, s.workspace, s.workspace_bytes = 4, 128, FAKE, L.sf_workspace_bytes(ctx, 4, 4, 128)
    assert commit() == sfb.SF_ESTATE
    assert L.sf_last_hip_error(ctx) == 0
    L.sf_destroy(ctx)


def test_oracle_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3], np.float32))
    np.testing.assert_allclose(so.kept_weights(l) * 0.4, [0.1, 0.4, 0.2, 0.3], rtol=1e-6)
    assert list(so.kept_weights(l, top_k=2) > 0) == [False, True, False, True]
    assert list(so.kept_weights(l, top_p=0.75) > 0) == [False, True, True, True]      # 0.4 + 0.3 < 0.75
    assert list(so.kept_weights(l, top_p=0.65) > 0) == [False, True, False, True]
    assert list(so.kept_weights(l, min_p=0.45) > 0) == [False, True, True, True]
    assert list(so.kept_weights(l, temperature=0) > 0) == [False, True, False, False]
    w = so.kept_weights(l)
    assert [so.draw(w, u) for u in (0.0, 0.05, 0.2, 0.6, 0.9, 0.999)] == [0, 0, 1, 2, 3, 3]
    ties = np.zeros(4, np.float32)
    assert list(so.kept_weights(ties, top_k=2)) == [1, 1, 0, 0]
    assert list(so.kept_weights(ties, top_p=0.5)) == [1, 1, 0, 0]
    assert list(so.kept_weights(ties, top_p=0.51)) == [1, 1, 1, 0]
    # acceptance: p(d) = 0.4, q(d) = 1 for a certain draft
    target = np.stack([l, l])
    assert so.accept([1], target, [0.39], 0.0, (1.0, 0, 1.0, 0.0))[:2] == (1, 0)
    n, token, rest = so.accept([1], target, [0.41], 0.4, (1.0, 0, 1.0, 0.0))
    assert n == 0 and token == 2 and rest[1] == 0


def test_engine_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    from paper_2511_20340_amd.engine import Engine
    eng = Engine.__new__(Engine)                            # the checks come before anything on a device
    eng.dev, eng.B, eng.V = torch.device("cuda", 0), 2, 10
    x, u = torch.zeros(3, 10), torch.zeros(3)
    for bad in ((x, u), (x.double(), u), (x[:, ::2], u), (x[0], u), (x, torch.zeros(4))):
        with pytest.raises(ValueError):
            eng.sf_op_sample(*bad)
    with pytest.raises(ValueError):
        eng.sf_op_sample(x, u, group=0)
    with pytest.raises(ValueError):
        eng.sf_op_accept_sampled(1, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 2, 10), torch.zeros(2, 1), torch.zeros(2))
