"""Refusals of the shared-prefix attention, on the host: status codes before anything is launched."""
import ctypes as C

from paper_2511_20340_amd import binding as sfb
from test_abi import cfg, create

FAKE = 0x10000


def test_prefix_attention_validates_before_launching_anything():
    L = sfb.lib()
    bf = dict(dtype=sfb.SF_BF16, n_q_heads=8, n_kv_heads=2, head_dim=64, d_model=512)
    st, ctx = create(cfg(**bf), cfg(n_layers=1, **bf))
    assert st == sfb.SF_OK
    need = L.sf_prefix_attention_workspace_bytes(ctx, 4, 5, 1000, 100)
    assert need > 0 and need % 256 == 0
    for bad in ((0, 5, 1000, 100), (4, 0, 1000, 100), (4, 5, -1, 100), (4, 5, 1000, -1), (1 << 20, 2, 1000, 100)):
        assert L.sf_prefix_attention_workspace_bytes(ctx, *bad) == 0
    assert L.sf_prefix_attention_workspace_bytes(ctx, 4, 5, 0, 4000) == L.sf_attention_workspace_bytes(ctx, 4, 5, 4000)

    def call(**kw):
        a = dict(ctx=ctx, q=FAKE, pk=FAKE, pv=FAKE, P=1000, pcap=1024, kc=FAKE, vc=FAKE, kv=FAKE, B=4, n_q=5, cap=128,
                 mask=sfb.SF_MASK_CAUSAL, upper=100, out=FAKE, ws=FAKE, nb=need)
        a.update(kw)
        return L.sf_op_prefix_attention(a["ctx"], a["q"], a["pk"], a["pv"], a["P"], a["pcap"], a["kc"], a["vc"], a["kv"], a["B"],
                                        a["n_q"], a["cap"], a["mask"], a["upper"], a["out"], a["ws"], a["nb"], None)
    for bad in (dict(ctx=None), dict(q=None), dict(pk=None), dict(pv=None), dict(kc=None), dict(vc=None), dict(kv=None), dict(out=None),
                dict(B=0), dict(n_q=0), dict(cap=100), dict(cap=0), dict(mask=2), dict(upper=-1), dict(P=-1), dict(pcap=1000),
                dict(pcap=0), dict(q=FAKE + 8), dict(pk=FAKE + 2), dict(out=FAKE + 4)):
        assert call(**bad) == sfb.SF_EINVAL, bad
    assert call(upper=124) == sfb.SF_ECAPACITY             # 124 + 5 > 128
    assert call(P=1025) == sfb.SF_ECAPACITY                # more keys than the cache has room for
    assert call(nb=need - 1) == sfb.SF_ECAPACITY
    assert call(ws=None) == sfb.SF_ECAPACITY
    assert call(ws=FAKE + 16) == sfb.SF_ECAPACITY
    assert call(n_q=257, cap=512) == sfb.SF_EUNSUPPORTED   # 4 query heads per kv head x 257 rows > 1024
    assert call(B=1 << 16) == sfb.SF_EUNSUPPORTED
    assert call(pcap=1 << 25) == sfb.SF_EUNSUPPORTED       # a slab of 4 GiB
    assert L.sf_last_hip_error(ctx) == 0
    L.sf_destroy(ctx)


def test_set_prefix_validates():
    L = sfb.lib()
    bf = dict(dtype=sfb.SF_BF16, n_q_heads=8, n_kv_heads=2, head_dim=64, d_model=512)
    st, ctx = create(cfg(**bf), cfg(n_layers=1, **bf))
    assert st == sfb.SF_OK
    assert L.sf_prefix_workspace_bytes(ctx, 5, 4, 128) == 0 and L.sf_prefix_workspace_bytes(ctx, 4, 5, 128) == 0
    assert L.sf_prefix_workspace_bytes(ctx, 4, 4, 100) == 0
    need = L.sf_prefix_workspace_bytes(ctx, 4, 4, 128)
    # room for any part of the batch, any block up to the largest, any prefix
    for B in (1, 2, 3, 4):
        for n_q in range(1, 6):
            for P in (1, 33, 700, 5000, 100000):
                assert L.sf_prefix_attention_workspace_bytes(ctx, B, n_q, P, 128 - n_q) <= need

    def call(**kw):
        a = dict(len=100, cap=128, tk=FAKE, tv=FAKE, dk=FAKE, dv=FAKE, workspace=FAKE, workspace_bytes=need)
        a.update(kw)
        return L.sf_set_prefix(ctx, C.byref(sfb.Prefix(**a)))
    assert call() == sfb.SF_OK and call(dk=None, dv=None) == sfb.SF_OK
    for bad in (dict(len=0), dict(len=-1), dict(cap=100), dict(cap=0), dict(tk=None), dict(tv=None), dict(dk=None), dict(dv=None),
                dict(tk=FAKE + 8), dict(workspace=None), dict(workspace=FAKE + 16)):
        assert call(**bad) == sfb.SF_EINVAL, bad
    assert call(len=129) == sfb.SF_ECAPACITY
    assert call(cap=1 << 25) == sfb.SF_EUNSUPPORTED
    # steps look at the workspace and at the draft caches before anything is launched
    tw, dw, s = sfb.TargetWeights(), sfb.DraftWeights(), sfb.State()
    arr = (C.c_void_p * 2)(FAKE, FAKE)
    for n, _ in sfb.TargetWeights._fields_:
        setattr(tw, n, arr if n not in ("embed", "lm_head", "final_norm") else FAKE)
    for n, _ in sfb.DraftWeights._fields_:
        setattr(dw, n, FAKE)
    assert L.sf_bind(ctx, C.byref(tw), C.byref(dw)) == sfb.SF_OK
    for n in ("tk", "tv", "dk", "dv", "kv_len", "pending", "hooks", "n_new", "cu_new"):
        setattr(s, n, FAKE)
    s.B, s.cap, s.workspace, s.workspace_bytes = 4, 128, FAKE, L.sf_workspace_bytes(ctx, 4, 4, 128)
    assert call(workspace_bytes=16) == sfb.SF_OK
    assert L.sf_verify_step(ctx, C.byref(s), 4, FAKE, 0, None, FAKE, None) == sfb.SF_ECAPACITY
    assert L.sf_draft_step(ctx, C.byref(s), 4, sfb.SF_MASK_BIDIR, 0, FAKE, None, None) == sfb.SF_ECAPACITY
    assert call(dk=None, dv=None) == sfb.SF_OK
    assert L.sf_draft_step(ctx, C.byref(s), 4, sfb.SF_MASK_BIDIR, 0, FAKE, None, None) == sfb.SF_ESTATE
    for last in (0, 1):                                              # before the block's verify and commit
        assert L.sf_prefill_step(ctx, C.byref(s), 4, FAKE, FAKE, 4, FAKE, 0, 4, 2, last, FAKE, FAKE, FAKE, FAKE, None) == sfb.SF_ESTATE
    assert call() == sfb.SF_OK
    two_stage = sfb.SF_MASK_BIDIR | sfb.SF_DRAFT_TWO_STAGE
    assert L.sf_draft_step(ctx, C.byref(s), 4, two_stage, 0, FAKE, None, None) == sfb.SF_EUNSUPPORTED
    assert L.sf_set_prefix(None, None) == sfb.SF_EINVAL and L.sf_set_prefix(ctx, None) == sfb.SF_OK
    assert L.sf_last_hip_error(ctx) == 0
    L.sf_destroy(ctx)
