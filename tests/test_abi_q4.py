"""Host-side argument checks of the page-table, rotary and 4-bit cache calls (no GPU:
every case fails before anything is launched)."""
import ctypes

import pytest

import paper_2603_19610_amd as pv

FAKE = ctypes.c_void_p(4096)     # never dereferenced
ODD = ctypes.c_void_p(4097)
NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


def _resize(**kw):
    a = dict(B=4, page=32, mp=8, np=64, len=FAKE, held=FAKE, table=FAKE, free=FAKE, nf=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    return pv.lib().pvlm_pages_resize(a["B"], a["page"], a["mp"], a["np"], a["len"], a["held"], a["table"], a["free"],
                                      a["nf"], None, None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(len=None), NULL), (dict(held=None), NULL), (dict(table=None), NULL), (dict(free=None), NULL),
    (dict(nf=None), NULL), (dict(B=0), SHAPE), (dict(page=48), SHAPE), (dict(page=16), SHAPE), (dict(mp=0), SHAPE),
    (dict(np=0), SHAPE), (dict(np=1 << 31), SHAPE), (dict(mp=(1 << 25) + 1), SHAPE), (dict(B=4097), UNSUPPORTED),
])
def test_resize_rejects(kw, code):
    assert _resize(**kw) == code


def _slots(**kw):
    a = dict(B=4, n=16, rps=0, page=32, mp=8, np=64, table=FAKE, ctx=FAKE, new=FAKE, slots=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    return pv.lib().pvlm_slot_map(a["B"], a["n"], a["rps"], a["page"], a["mp"], a["np"], a["table"], a["ctx"], a["new"],
                                  a["slots"], None, None, None, None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(ctx=None), NULL), (dict(new=None), NULL), (dict(slots=None), NULL), (dict(B=0), SHAPE), (dict(n=0), SHAPE),
    (dict(n=(1 << 30) + 1), SHAPE), (dict(rps=-1), SHAPE), (dict(rps=3), SHAPE), (dict(page=33), SHAPE),
    (dict(page=0), SHAPE), (dict(table=None), SHAPE), (dict(table=None, mp=1, page=(1 << 30) + 1), SHAPE),
    (dict(mp=0), SHAPE), (dict(np=0), SHAPE), (dict(np=1 << 31), SHAPE), (dict(B=4097), UNSUPPORTED),
    (dict(slots=ODD), UNSUPPORTED),
])
def test_slot_map_rejects(kw, code):
    assert _slots(**kw) == code


def _params(**kw):
    p = dict(base=1e4, factor=1.0, orig_ctx=0.0, alpha=0.0, beta=0.0, mscale=1.0, rot_dim=64, layout=0, scaling=0,
             sections=(0, 0, 0))
    p.update(kw)
    p["sections"] = (ctypes.c_int32 * 3)(*p["sections"])
    return pv.RotaryParams(*p.values())


def _rotary(q4=False, rot=None, **kw):
    a = dict(dt=1, N=6, Hq=8, Hkv=2, D=128, pos=FAKE, q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, slots=FAKE, nb=2,
             br=64, qo=FAKE, kc=FAKE, ke=FAKE, vc=FAKE, ve=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    p = ctypes.byref(_params(**rot)) if rot is not None else ctypes.byref(_params())
    head = (a["dt"], a["N"], a["Hq"], a["Hkv"], a["D"], p if rot != {"null": 1} else None, a["pos"], a["q"], a["qs"],
            a["k"], a["ks"], a["v"], a["vs"], a["slots"], a["nb"], a["br"], a["qo"])
    if q4:
        return pv.lib().pvlm_rotary_append_q4(*head, a["kc"], a["ke"], a["vc"], a["ve"], None, None)
    return pv.lib().pvlm_rotary_append(*head, a["kc"], a["vc"], None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(pos=None), NULL), (dict(q=None), NULL), (dict(slots=None), NULL), (dict(qo=None), NULL), (dict(kc=None), NULL),
    (dict(vc=None), NULL), (dict(dt=2), UNSUPPORTED), (dict(N=0), SHAPE), (dict(N=1 << 24), SHAPE), (dict(Hkv=3), SHAPE),
    (dict(Hq=0), SHAPE), (dict(nb=0), SHAPE), (dict(br=0), SHAPE), (dict(br=(1 << 30) + 1), SHAPE), (dict(nb=1 << 31), SHAPE),
    (dict(qs=1016), SHAPE), (dict(ks=0), SHAPE), (dict(vs=(1 << 40) + 8), SHAPE), (dict(qs=1028), UNSUPPORTED),
    (dict(vs=257), UNSUPPORTED), (dict(q=ODD), UNSUPPORTED), (dict(kc=ODD), UNSUPPORTED), (dict(qo=ODD), UNSUPPORTED),
    (dict(slots=ODD), UNSUPPORTED), (dict(Hq=65536, Hkv=1, qs=1 << 30), SHAPE),
    (dict(rot=dict(rot_dim=136)), SHAPE), (dict(rot=dict(rot_dim=60)), SHAPE), (dict(rot=dict(layout=2)), SHAPE),
    (dict(rot=dict(scaling=4)), SHAPE), (dict(rot=dict(base=0.5)), SHAPE), (dict(rot=dict(scaling=1, factor=-1.0)), SHAPE),
    (dict(rot=dict(sections=(16, 8, 9))), SHAPE), (dict(rot=dict(sections=(-8, 32, 8))), SHAPE),
    (dict(rot=dict(mscale=float("inf"))), SHAPE),
])
def test_rotary_rejects(kw, code):
    assert _rotary(**kw) == code
    assert _rotary(q4=True, **kw) == code


def test_rotary_limits_of_each_cache():
    assert _rotary(D=12, qs=96, ks=24, vs=24) == SHAPE and _rotary(D=264, qs=4096, ks=1024, vs=1024) == SHAPE
    assert _rotary(q4=True, D=96) == UNSUPPORTED and _rotary(q4=True, dt=0) == UNSUPPORTED
    assert _rotary(q4=True, ke=None) == NULL and _rotary(q4=True, ve=ODD) == UNSUPPORTED
    assert pv.lib().pvlm_rotary_freqs(None, None) == NULL


def _quantize(paged=False, **kw):
    a = dict(dt=1, L=2, B=1, Hkv=2, D=128, src=50, k=FAKE, v=FAKE, len=FAKE, n_cap=64, kc=FAKE, ke=FAKE, vc=FAKE,
             ve=FAKE, page=32, mp=2, np=4, table=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    L = pv.lib()
    out = (a["kc"], a["ke"], a["vc"], a["ve"], None, None)
    if paged:
        return L.pvlm_quantize_kv_q4_paged(a["dt"], a["L"], a["B"], a["Hkv"], a["D"], a["page"], a["mp"], a["np"],
                                           a["src"], a["k"], a["v"], a["len"], a["table"], *out)
    return L.pvlm_quantize_kv_q4(a["dt"], a["L"], a["B"], a["Hkv"], a["D"], a["src"], a["k"], a["v"], a["len"],
                                 a["n_cap"], *out)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), NULL), (dict(len=None), NULL), (dict(vc=None), NULL), (dict(dt=2), UNSUPPORTED),
    (dict(dt=3), UNSUPPORTED), (dict(D=32), UNSUPPORTED), (dict(src=0), SHAPE), (dict(L=0), SHAPE), (dict(L=65536), SHAPE),
    (dict(Hkv=65536), SHAPE), (dict(n_cap=40), SHAPE), (dict(k=ODD), UNSUPPORTED), (dict(ke=ODD), UNSUPPORTED),
    (dict(src=(1 << 30) + 1), SHAPE),
])
def test_quantize_rejects(kw, code):
    assert _quantize(**kw) == code
    if "n_cap" not in kw:
        assert _quantize(paged=True, **kw) == code
    assert _quantize(paged=True, table=None) == NULL
    assert _quantize(paged=True, page=33) == SHAPE


def _verify(paged=False, **kw):
    a = dict(dt=1, B=1, T=5, Hq=8, Hkv=2, D=128, n_cap=128, max_ctx=100, scale=0.088, q=FAKE, kc=FAKE, ke=FAKE,
             vc=FAKE, ve=FAKE, ctx=FAKE, out=FAKE, ws=FAKE, wsb=1 << 40, page=32, mp=4, np=8, table=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    L = pv.lib()
    cache = (a["kc"], a["ke"], a["vc"], a["ve"])
    out = (a["ctx"], a["out"], None, None, a["ws"], a["wsb"], None, None)
    head = (a["dt"], a["B"], a["T"], a["Hq"], a["Hkv"], a["D"])
    if paged:
        return L.pvlm_verify_attn_q4_paged(*head, a["page"], a["mp"], a["np"], a["max_ctx"], a["scale"], a["q"],
                                           *cache, a["table"], *out)
    return L.pvlm_verify_attn_q4(*head, a["n_cap"], a["max_ctx"], a["scale"], a["q"], *cache, *out)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(ctx=None), NULL), (dict(out=None), NULL), (dict(ke=None), NULL),
    (dict(T=0), SHAPE), (dict(B=0), SHAPE), (dict(max_ctx=124), SHAPE), (dict(max_ctx=-1), SHAPE),
    (dict(n_cap=130), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(Hkv=3), UNSUPPORTED), (dict(T=33), UNSUPPORTED), (dict(dt=0), UNSUPPORTED),
    (dict(dt=3), UNSUPPORTED), (dict(Hq=128, Hkv=1, T=9, max_ctx=90), UNSUPPORTED),
    (dict(B=1 << 20), SHAPE), (dict(kc=ODD), UNSUPPORTED), (dict(ve=ODD), UNSUPPORTED),
    (dict(q=ODD), UNSUPPORTED),
])
def test_verify_rejects(kw, code):
    assert _verify(**kw) == code
    if "n_cap" not in kw:
        assert _verify(paged=True, **kw) == code


def test_verify_paged_rejects():
    assert _verify(paged=True, table=None) == NULL
    for bad in (dict(page=48), dict(page=1 << 21), dict(mp=0), dict(np=0)):
        assert _verify(paged=True, **bad) == SHAPE
    assert _verify(paged=True, mp=3) == SHAPE      # 96 logical rows < max_ctx + T


def _gather(paged=False, **kw):
    a = dict(dt=3, L=2, B=1, Hkv=2, D=128, n_cap=64, kc=FAKE, ke=FAKE, vc=FAKE, ve=FAKE, idx=FAKE, k=FAKE, k_cap=4,
             tb=FAKE, tl=FAKE, cap=32, kd=FAKE, kde=FAKE, vd=FAKE, vde=FAKE, page=32, mp=2, np=4, table=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    L = pv.lib()
    cache = (a["kc"], a["ke"], a["vc"], a["ve"])
    tail = (a["idx"], a["k"], a["k_cap"], a["tb"], a["tl"], a["cap"], 0, a["kd"], a["kde"], a["vd"], a["vde"],
            None, None)
    head = (a["dt"], a["L"], a["B"], a["Hkv"], a["D"])
    if paged:
        return L.pvlm_gather_kv_q4_paged(*head, a["page"], a["mp"], a["np"], *cache, a["table"], *tail)
    return L.pvlm_gather_kv_q4(*head, a["n_cap"], *cache, *tail)


@pytest.mark.parametrize("kw,code", [
    (dict(kc=None), NULL), (dict(k=None), NULL), (dict(idx=None), NULL), (dict(tl=None), NULL),
    (dict(kd=None), NULL), (dict(vde=None), NULL), (dict(dt=2), UNSUPPORTED), (dict(D=256), UNSUPPORTED),
    (dict(cap=33), SHAPE), (dict(cap=0), SHAPE), (dict(cap=-1, dt=1), SHAPE), (dict(k_cap=-1), SHAPE),
    (dict(n_cap=48), SHAPE), (dict(L=70000), SHAPE), (dict(kd=ODD), UNSUPPORTED), (dict(kd=ODD, dt=1), UNSUPPORTED),
])
def test_gather_rejects(kw, code):
    assert _gather(**kw) == code
    if "n_cap" not in kw:
        assert _gather(paged=True, **kw) == code
    assert _gather(dt=1, cap=0, kde=None, vde=None) == 0          # nothing to do, nothing launched
    assert _gather(paged=True, table=None) == NULL


def test_calls_of_other_types_do_not_take_the_4bit_type():
    L = pv.lib()
    assert L.pvlm_verify_attn(pv.PVLM_E2M1, 1, 5, 8, 2, 128, 100, 95, 0.088, FAKE, FAKE, FAKE, FAKE, FAKE, None,
                              None, FAKE, 1 << 30, None, None) == UNSUPPORTED
    assert L.pvlm_gather_kv(pv.PVLM_E2M1, 1, 1, 1, 128, 10, FAKE, FAKE, FAKE, FAKE, 4, FAKE, FAKE, 8, FAKE, FAKE,
                            None, None) == UNSUPPORTED
