"""Refusals of the shared-prefix attention, on the host: status codes before anything is launched."""
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
