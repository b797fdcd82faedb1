"""Host-side argument checks of the 8-bit cache calls (no GPU: every case fails
before anything is launched), and the plan of verify over them."""
import ctypes

import pytest

import paper_2603_19610_amd as pv

FAKE = ctypes.c_void_p(4096)     # never dereferenced
ODD = ctypes.c_void_p(4097)
NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


def _append(paged=False, **kw):
    a = dict(dt=1, B=1, T=4, Hq=8, Hkv=2, D=128, n_cap=64, base=1e6, sec=None, pos=FAKE, q=FAKE, k=FAKE,
             v=FAKE, ctx=FAKE, qo=FAKE, kc=FAKE, ke=FAKE, vc=FAKE, ve=FAKE, page=32, mp=2, np=4, table=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    L = pv.lib()
    head = (a["dt"], a["B"], a["T"], a["Hq"], a["Hkv"], a["D"])
    rows = (a["pos"], a["q"], a["k"], a["v"])
    out = (a["ctx"], a["qo"], a["kc"], a["ke"], a["vc"], a["ve"], None, None)
    if paged:
        return L.pvlm_rope_append_q8_paged(*head, a["page"], a["mp"], a["np"], a["base"], a["sec"], *rows,
                                           a["table"], *out)
    return L.pvlm_rope_append_q8(*head, a["n_cap"], a["base"], a["sec"], *rows, *out)


def _sections(*s):
    return (ctypes.c_int32 * 3)(*s)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(ctx=None), NULL), (dict(kc=None), NULL), (dict(ve=None), NULL),
    (dict(qo=None), NULL), (dict(dt=0), UNSUPPORTED), (dict(dt=2), UNSUPPORTED), (dict(D=96), UNSUPPORTED),
    (dict(T=0), SHAPE), (dict(B=0), SHAPE), (dict(Hkv=3), SHAPE), (dict(n_cap=65), SHAPE), (dict(n_cap=0), SHAPE),
    (dict(T=65), SHAPE), (dict(base=1.0), SHAPE), (dict(base=float("nan")), SHAPE),
    (dict(sec=_sections(16, 24, 25)), SHAPE), (dict(sec=_sections(-1, 41, 24)), SHAPE),
    (dict(kc=ODD), UNSUPPORTED), (dict(ve=ODD), UNSUPPORTED), (dict(q=ODD), UNSUPPORTED),
    (dict(B=1 << 19, T=32), SHAPE), (dict(Hq=65535, Hkv=1), SHAPE),
])
def test_append_rejects(kw, code):
    assert _append(**kw) == code
    if "n_cap" not in kw:
        assert _append(paged=True, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), NULL), (dict(page=48), SHAPE), (dict(page=16), SHAPE), (dict(mp=0), SHAPE),
    (dict(np=0), SHAPE), (dict(np=1 << 31), SHAPE),
])
def test_append_paged_rejects(kw, code):
    assert _append(paged=True, **kw) == code


def _quantize(paged=False, **kw):
    a = dict(dt=1, L=2, B=1, Hkv=2, D=128, src=50, k=FAKE, v=FAKE, len=FAKE, n_cap=64, kc=FAKE, ke=FAKE, vc=FAKE,
             ve=FAKE, page=32, mp=2, np=4, table=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    L = pv.lib()
    out = (a["kc"], a["ke"], a["vc"], a["ve"], None, None)
    if paged:
        return L.pvlm_quantize_kv_paged(a["dt"], a["L"], a["B"], a["Hkv"], a["D"], a["page"], a["mp"], a["np"],
                                        a["src"], a["k"], a["v"], a["len"], a["table"], *out)
    return L.pvlm_quantize_kv(a["dt"], a["L"], a["B"], a["Hkv"], a["D"], a["src"], a["k"], a["v"], a["len"],
                              a["n_cap"], *out)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), NULL), (dict(len=None), NULL), (dict(vc=None), NULL), (dict(dt=2), UNSUPPORTED),
    (dict(D=32), UNSUPPORTED), (dict(src=0), SHAPE), (dict(L=0), SHAPE), (dict(L=65536), SHAPE),
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
        return L.pvlm_verify_attn_q8_paged(*head, a["page"], a["mp"], a["np"], a["max_ctx"], a["scale"], a["q"],
                                           *cache, a["table"], *out)
    return L.pvlm_verify_attn_q8(*head, a["n_cap"], a["max_ctx"], a["scale"], a["q"], *cache, *out)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(ctx=None), NULL), (dict(out=None), NULL), (dict(ke=None), NULL),
    (dict(T=0), SHAPE), (dict(B=0), SHAPE), (dict(max_ctx=124), SHAPE), (dict(max_ctx=-1), SHAPE),
    (dict(n_cap=130), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(Hkv=3), UNSUPPORTED), (dict(T=33), UNSUPPORTED), (dict(dt=0), UNSUPPORTED),
    (dict(dt=2), UNSUPPORTED), (dict(Hq=128, Hkv=1, T=9, max_ctx=90), UNSUPPORTED),
    (dict(B=1 << 20), SHAPE), (dict(kc=ODD), UNSUPPORTED), (dict(ve=ODD), UNSUPPORTED), (dict(q=ODD), UNSUPPORTED),
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
    a = dict(dt=2, L=2, B=1, Hkv=2, D=128, n_cap=64, kc=FAKE, ke=FAKE, vc=FAKE, ve=FAKE, idx=FAKE, k=FAKE, k_cap=4,
             tb=FAKE, tl=FAKE, cap=32, kd=FAKE, kde=FAKE, vd=FAKE, vde=FAKE, page=32, mp=2, np=4, table=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    L = pv.lib()
    cache = (a["kc"], a["ke"], a["vc"], a["ve"])
    tail = (a["idx"], a["k"], a["k_cap"], a["tb"], a["tl"], a["cap"], 0, a["kd"], a["kde"], a["vd"], a["vde"],
            None, None)
    head = (a["dt"], a["L"], a["B"], a["Hkv"], a["D"])
    if paged:
        return L.pvlm_gather_kv_q8_paged(*head, a["page"], a["mp"], a["np"], *cache, a["table"], *tail)
    return L.pvlm_gather_kv_q8(*head, a["n_cap"], *cache, *tail)


@pytest.mark.parametrize("kw,code", [
    (dict(kc=None), NULL), (dict(k=None), NULL), (dict(idx=None), NULL), (dict(tl=None), NULL),
    (dict(kd=None), NULL), (dict(vde=None), NULL), (dict(dt=3), UNSUPPORTED), (dict(D=256), UNSUPPORTED),
    (dict(cap=33), SHAPE), (dict(cap=0), SHAPE), (dict(cap=-1, dt=1), SHAPE), (dict(k_cap=-1), SHAPE),
    (dict(n_cap=48), SHAPE), (dict(L=70000), SHAPE), (dict(kd=ODD), UNSUPPORTED), (dict(kd=ODD, dt=1), UNSUPPORTED),
])
def test_gather_rejects(kw, code):
    assert _gather(**kw) == code
    if "n_cap" not in kw:
        assert _gather(paged=True, **kw) == code
    assert _gather(dt=1, cap=0, kde=None, vde=None) == 0          # nothing to do, nothing launched
    assert _gather(paged=True, table=None) == NULL


def test_calls_of_other_types_do_not_take_the_8bit_type():
    L = pv.lib()
    assert L.pvlm_verify_attn(pv.PVLM_E4M3, 1, 5, 8, 2, 128, 100, 95, 0.088, FAKE, FAKE, FAKE, FAKE, FAKE, None,
                              None, FAKE, 1 << 30, None, None) == UNSUPPORTED
    assert L.pvlm_gather_kv(pv.PVLM_E4M3, 1, 1, 1, 128, 10, FAKE, FAKE, FAKE, FAKE, 4, FAKE, FAKE, 8, FAKE, FAKE,
                            None, None) == UNSUPPORTED
