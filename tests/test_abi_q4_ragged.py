"""Host-side argument checks of the ragged 4-bit verify (no GPU: every case fails before
anything is launched)."""
import pytest

import paper_2603_19610_amd as pv
from test_abi_q4 import FAKE, NULL, ODD, SHAPE, UNSUPPORTED


def _verify(paged=False, **kw):
    a = dict(dt=1, B=1, T=5, Hq=8, Hkv=2, D=128, n_cap=128, max_ctx=100, scale=0.088, q=FAKE, kc=FAKE, ke=FAKE,
             vc=FAKE, ve=FAKE, ctx=FAKE, new=FAKE, out=FAKE, ws=FAKE, wsb=1 << 40, page=32, mp=4, np=8, table=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    L = pv.lib()
    cache = (a["kc"], a["ke"], a["vc"], a["ve"])
    out = (a["ctx"], a["new"], a["out"], None, None, a["ws"], a["wsb"], None, None)
    head = (a["dt"], a["B"], a["T"], a["Hq"], a["Hkv"], a["D"])
    if paged:
        return L.pvlm_verify_attn_q4_ragged_paged(*head, a["page"], a["mp"], a["np"], a["max_ctx"], a["scale"], a["q"],
                                                  *cache, a["table"], *out)
    return L.pvlm_verify_attn_q4_ragged(*head, a["n_cap"], a["max_ctx"], a["scale"], a["q"], *cache, *out)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(ctx=None), NULL), (dict(out=None), NULL), (dict(ke=None), NULL), (dict(T=0), SHAPE),
    (dict(max_ctx=124), SHAPE), (dict(scale=0.0), SHAPE), (dict(D=96), UNSUPPORTED), (dict(T=33), UNSUPPORTED),
    (dict(dt=0), UNSUPPORTED), (dict(B=1 << 20), SHAPE), (dict(ve=ODD), UNSUPPORTED), (dict(q=ODD), UNSUPPORTED),
])
@pytest.mark.parametrize("new", [FAKE, None])
def test_ragged_verify_rejects(kw, code, new):
    assert _verify(new=new, **kw) == code and _verify(paged=True, new=new, **kw) == code


def test_ragged_verify_paged_rejects():
    assert _verify(paged=True, table=None) == NULL
    for bad in (dict(page=48), dict(mp=0), dict(np=0), dict(mp=3)):
        assert _verify(paged=True, **bad) == SHAPE
