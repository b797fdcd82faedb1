"""GPU parity of the page-table and slot calls (exact: whole numbers), and of the
rotary append: its rotation within the rounding of its type, its copies bit for bit."""
import random

import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
from gpu_util import note
from oracle import pages as G
from oracle import quant4 as Q
from oracle import rotary as R
from oracle.quant import bf16 as to_bf16
from test_parity_q4 import check_all, empty_cache, host, i32, values
from test_parity_q8 import cap32, dev, queries, rows_like_a_models, status_word

pytestmark = pytest.mark.gpu


class Pool:
    """The device's state of a batch's pages beside the oracle's."""

    def __init__(self, B, P, max_pages, n_pages, seed=0):
        self.P = P
        order = list(range(n_pages))
        random.Random(seed).shuffle(order)
        self.held, self.table, self.stack = [0] * B, [[-1] * max_pages for _ in range(B)], order
        free = torch.full((n_pages,), -7, dtype=torch.int32)
        free[:] = torch.tensor(order)
        self.d = [i32(self.held), i32(self.table), free.cuda(), i32([n_pages])]

    def resize(self, length, status=None):
        granted = pv.pages_resize(i32(length), *self.d, page_size=self.P, status=status)
        want = G.resize(length, self.held, self.table, self.stack, self.P)
        torch.cuda.synchronize()
        assert granted.tolist() == want
        held, table, free, n_free = self.d
        assert held.tolist() == self.held and table.tolist() == self.table
        assert n_free.item() == len(self.stack) and free[:len(self.stack)].tolist() == self.stack
        return want


@pytest.mark.parametrize("B,P,max_pages,n_pages", [
    (1, 32, 1, 1), (1, 32, 700, 900), (3, 64, 40, 70), (16, 32, 300, 2500), (17, 256, 9, 80), (64, 32, 30, 1200),
    (300, 1024, 5, 900), (1500, 32, 12, 9000), (4096, 32, 3, 9000), (2, 1 << 20, 4, 5),
])
def test_resize_grows_and_cuts_like_the_oracle(B, P, max_pages, n_pages):
    rng = np.random.default_rng(B + P)
    pool = Pool(B, P, max_pages, n_pages, seed=B)
    most = P * max_pages
    st = status_word()
    steps = [rng.integers(0, most + 1, B), rng.integers(0, most // 3 + 1, B), np.full(B, most), np.zeros(B, int),
             np.full(B, 1), rng.integers(0, most + 1, B), rng.integers(0, most + 1, B)]
    short = False
    for i, length in enumerate(steps):
        note(f"resize B{B} P{P} pages {max_pages} of {n_pages}, step {i}")
        short |= 0 in pool.resize([int(x) for x in length], status=st)
    assert int(st.item()) == (pv.PVLM_DEV_NO_PAGES if short else 0)


def test_resize_flags_and_survives_a_state_that_makes_no_sense():
    """Lengths, counts and entries out of range are clamped or dropped; nothing leaves the tensors."""
    P, max_pages, n_pages = 32, 4, 10
    guard = 123456

    def run(length, held, table, free, n_free):
        st = status_word()
        big = torch.full((len(held) * max_pages + 64,), guard, dtype=torch.int32, device="cuda")
        t = big[32:-32].view(len(held), max_pages)
        t.copy_(i32(table))
        bigf = torch.full((n_pages + 64,), guard, dtype=torch.int32, device="cuda")
        f = bigf[32:-32]
        f.copy_(i32(free))
        d = [i32(held), t, f, i32([n_free])]
        granted = pv.pages_resize(i32(length), *d, page_size=P, status=st)
        torch.cuda.synchronize()
        for g in (big, bigf):
            assert bool((g[:32] == guard).all()) and bool((g[-32:] == guard).all())
        return int(st.item()), granted.tolist(), d
    note("resize: lengths, held and free counts out of range")
    empty, stack = [[-1] * 4] * 2, list(range(10))
    flags, granted, d = run([-5, 4 * P + 1], [0, 0], empty, stack, 10)
    assert flags == pv.PVLM_DEV_RANGE and granted == [1, 1] and d[0].tolist() == [0, 4] and d[3].item() == 6
    flags, granted, d = run([P, P], [-3, 9], [[-1] * 4, [1, 2, 3, 4]], stack, 0)
    assert flags == pv.PVLM_DEV_RANGE and granted == [1, 1] and d[0].tolist() == [1, 1]
    flags, _, d = run([P, 0], [0, 0], empty, stack, 99)
    assert flags == pv.PVLM_DEV_RANGE and d[3].item() == 9 and d[1][0, 0].item() == 9
    flags, granted, d = run([P, 0], [0, 0], empty, stack, -1)
    assert flags == pv.PVLM_DEV_RANGE | pv.PVLM_DEV_NO_PAGES and granted == [0, 1] and d[3].item() == 0
    # entries that name no page are dropped, the others keep their order
    flags, _, d = run([0, 0], [4, 2], [[5, -1, 99, 6], [7, 10, 0, 0]], [1, 2, 0, 0, 0, 0, 0, 0, 0, 0], 2)
    assert flags == pv.PVLM_DEV_RANGE and d[3].item() == 5 and d[2][:5].tolist() == [1, 2, 5, 6, 7]
    assert d[1].tolist() == [[-1] * 4, [-1, -1, 0, 0]]
    # more pages come back than the stack has room for
    flags, _, d = run([0, 0], [4, 4], [[0, 1, 2, 3], [4, 5, 6, 7]], stack, 5)
    assert flags == pv.PVLM_DEV_RANGE and d[3].item() == 10 and d[2].tolist() == [0, 1, 2, 3, 4, 0, 1, 2, 3, 4]


@pytest.mark.parametrize("B,P,ctx_hi,new_hi,extra", [(1, 32, 0, 1, 0), (1, 64, 9000, 5000, 7), (5, 32, 100, 40, 0),
                                                    (64, 32, 3000, 9, 100), (777, 32, 300, 3, 1), (4096, 32, 64, 2, 0)])
def test_slot_map(B, P, ctx_hi, new_hi, extra):
    rng = np.random.default_rng(B)
    ctx, new = rng.integers(0, ctx_hi + 1, B), rng.integers(0, new_hi + 1, B)
    new[0] = new_hi
    if B > 4:
        new[1:3] = 0                           # empty sequences between others
    ctx, new = ctx.tolist(), new.tolist()
    max_pages = -(-(ctx_hi + new_hi) // P) + 1
    n_pages = B * max_pages + 5
    table = rng.permutation(n_pages)[:B * max_pages].reshape(B, max_pages)
    t = i32(table.tolist())
    for rps, tab in ((0, t), (new_hi, t), (0, None), (new_hi + 2, None)):
        n_rows = B * rps if rps else sum(new) + extra
        page, pages = (P, n_pages) if tab is not None else (ctx_hi + new_hi + 3, B)
        note(f"slot map B{B} P{page} rows {n_rows} apart {rps} padded {tab is None}")
        st = status_word()
        got = pv.slot_map(i32(ctx), i32(new), n_rows, page_size=page, n_pages=pages, page_table=tab, rows_per_seq=rps,
                          status=st)
        want = G.slot_map(ctx, new, n_rows, page, None if tab is None else table, rps)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        for name, a, b in zip(("slots", "pos", "seq", "start"), got, want):
            assert a.cpu().numpy().tolist() == [int(x) for x in b], name
    only = pv.slot_map(i32(ctx), i32(new), max(sum(new), 1), page_size=P, n_pages=n_pages, page_table=t, want_pos=False,
                       want_seq=False, want_start=False)
    assert only[1:] == (None, None, None)


def test_slot_map_flags_what_has_no_slot():
    t = i32([[3, 99, -1], [0, 1, 2]])
    run = lambda ctx, new, n, **kw: (lambda st: ([x.tolist() for x in pv.slot_map(
        i32(ctx), i32(new), n, page_size=32, n_pages=10, page_table=t, status=st, **kw)], int(st.item())))(status_word())
    note("slot map: bad entries, lengths past the table, counts out of range")
    (s, p, q, _), f = run([30, 0], [4, 1], 5)
    assert f == 1 and s == [126, 127, -1, -1, 0] and p == [30, 31, 0, 0, 0] and q == [0, 0, 0, 0, 1]
    (s, _, _, _), f = run([95, 0], [2, 1], 3)
    assert f == 1 and s == [-1, -1, 0]
    (s, _, _, _), f = run([-1, 0], [2, 1], 3)
    assert f == 1 and s == [-1, -1, 0]
    (s, _, _, start), f = run([0, 0], [2, 3], 4)              # one row more than there is room for
    assert f == 1 and s == [96, 97, 0, 1] and start == [0, 2, 4]
    (s, _, _, start), f = run([0, 0], [-2, 3], 4)
    assert f == 1 and s == [0, 1, 2, -1] and start == [0, 0, 3]
    (s, _, _, _), f = run([0, 0], [3, 1], 4, rows_per_seq=2)
    assert f == 1 and s == [96, 97, 0, -1]
    (s, _, _, _), f = run([0, 0], [0, 0], 3)
    assert f == 0 and s == [-1, -1, -1]


# ------------------------------------------------------------------ rotary --
ROTS = [
    dict(rot_dim=128, base=1e6), dict(rot_dim=64, base=1e4, layout="interleaved"),
    dict(rot_dim=32, base=1e4, scaling="linear", factor=4.0), dict(rot_dim=8, base=500.0, layout="interleaved"),
    dict(rot_dim=64, base=1e6, scaling="yarn", factor=4.0, orig_ctx=32768.0, alpha=1.0, beta=32.0, mscale=1.1386),
    dict(rot_dim=64, base=5e5, layout="interleaved", scaling="parts", factor=8.0, orig_ctx=8192.0, alpha=1.0, beta=4.0),
    dict(rot_dim=64, base=1e6, sections=(8, 12, 12)),
    dict(rot_dim=48, base=1e6, sections=(8, 8, 8), layout="interleaved"),
]


def turned(x, pos, rot):
    f = R.frequencies(rot["rot_dim"], rot["base"], **{k: rot[k] for k in ("scaling", "factor", "orig_ctx", "alpha", "beta")
                                                     if k in rot})
    return R.rotate(x, pos, f, rot.get("layout", "half"), rot.get("mscale", 1.0), rot.get("sections"))


def fused_rows(rng, N, Hq, Hkv, D, dtype, pad=0):
    """q, k and v as slices of one projection's rows."""
    x = dev(rows_like_a_models(rng, (N, Hq + 2 * Hkv, D))).to(dtype)
    if pad:
        x = torch.cat([x.flatten(1), torch.full((N, pad), float("nan"), dtype=dtype, device="cuda")], dim=1)
        x = x[:, :-pad].unflatten(1, (Hq + 2 * Hkv, D))
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rot", ROTS, ids=lambda r: f"{r['rot_dim']}{r.get('layout', '')}{r.get('scaling', '')}{'m' if 'sections' in r else ''}")
@pytest.mark.parametrize("N,Hq,Hkv,D,blocks,rows", [(1, 1, 1, 128, 1, 32), (7, 28, 4, 128, 9, 32), (300, 6, 2, 136, 5, 100),
                                                  (40, 3, 3, 256, 3, 1000)])
def test_rotary_append(dtype, rot, N, Hq, Hkv, D, blocks, rows):
    """A rotated value is off by one rounding of the float64 result to fp32 and one to its type (half a step each, 2^-24
    and 2^-9 + 2^-24 of it), and the angle: p f with p <= 200000 and a frequency off by 32 of 2^-53 turns by at most
    200000 * 34 * 2^-53 too far, so by 2^-30 of the pair's size.  Everything else is a copy."""
    rng = np.random.default_rng(N + D)
    q, k, v = fused_rows(rng, N, Hq, Hkv, D, dtype, pad=8 if N == 7 else 0)
    pos = rng.integers(0, 200000, (3, N)) if "sections" in rot else rng.integers(0, 200000, N)
    slots = rng.permutation(blocks * rows)[:N].astype(np.int64)
    if N > 4:
        slots[2], slots[N - 1] = -1, -9
    caches = [dev(rows_like_a_models(rng, (blocks, Hkv, rows, D))).to(dtype) for _ in range(2)]
    old = [c.clone() for c in caches]
    q_out = torch.full((N, Hq, D), 3.0, dtype=dtype, device="cuda")
    st = status_word()
    note(f"rotary {dtype} N{N} H{Hq}/{Hkv} D{D} {rot}")
    pv.rotary_append(q, k, v, dev(pos.astype(np.int32)), dev(slots), *caches, rotary=pv.Rotary(**rot), q_out=q_out, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    half = (2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24) + 2.0 ** -24
    real = slots >= 0

    def near(got, x):
        x = x.double().cpu().numpy()
        want, got, Rd = turned(x, pos, rot), got.double().cpu().numpy(), rot["rot_dim"]
        size = np.abs(x[..., :Rd]).max(axis=-1, keepdims=True) * 1.5 * rot.get("mscale", 1.0)
        assert np.all(np.abs(got - want)[..., :Rd] <= half * np.abs(want[..., :Rd]) + 2.0 ** -30 * size)
        assert np.array_equal(got[..., Rd:], x[..., Rd:])
    near(q_out[real], q[real]) if real.all() else None
    if not real.all():
        keep = np.flatnonzero(real)
        sub = lambda t: t[torch.from_numpy(keep).cuda()]
        full, pos = pos, pos[..., keep]
        near(sub(q_out), sub(q))
        assert bool((q_out[torch.from_numpy(np.flatnonzero(~real)).cuda()] == 3.0).all())
        k, v, slots = sub(k), sub(v), slots[keep]
    blk, r = torch.from_numpy(slots // rows).cuda(), torch.from_numpy(slots % rows).cuda()
    near(caches[0][blk, :, r], k)
    assert torch.equal(caches[1][blk, :, r], v)
    for c, o in zip(caches, old):
        c[blk, :, r] = o[blk, :, r]
        assert torch.equal(c, o)               # nothing else was touched


def test_rotary_equals_the_verify_rows_append():
    """The plain half layout gives what rope_append gives, to the last place of the angle's two ways."""
    rng = np.random.default_rng(2)
    B, T, Hq, Hkv, D, cap = 2, 9, 8, 2, 128, 1100
    q, kn, vn = (queries(rng, B, T, h, D) for h in (Hq, Hkv, Hkv))
    ctx = i32([1000, 13])
    pos = ctx[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
    a = [torch.zeros((B, Hkv, cap, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    b = [x.clone() for x in a]
    note("rotary against rope_append")
    q1 = pv.rope_append(q, kn, vn, pos, ctx, *a, base=1e6)
    slots, p, _, _ = pv.slot_map(ctx, i32([T] * B), B * T, page_size=cap, n_pages=B)
    assert torch.equal(p, pos.flatten())
    q2 = pv.rotary_append(q.flatten(0, 1), kn.flatten(0, 1), vn.flatten(0, 1), p, slots, *b, rotary=pv.Rotary(rot_dim=D, base=1e6))
    torch.cuda.synchronize()
    assert torch.equal(a[1], b[1])
    for x, y in ((q1.flatten(0, 1), q2), (a[0], b[0])):
        off = (x.float() - y.float()).abs()
        assert bool((off <= 2.0 ** -7 * x.float().abs()).all()) and (off > 0).float().mean().item() < 1e-3


@pytest.mark.parametrize("rot", ROTS[:2] + ROTS[4:7], ids=lambda r: f"{r['rot_dim']}{r.get('layout', '')}{r.get('scaling', '')}")
@pytest.mark.parametrize("N,Hq,Hkv,D,blocks,rows", [(1, 7, 1, 128, 2, 32), (16, 28, 4, 128, 30, 64), (501, 5, 5, 64, 3, 300),
                                                  (200, 64, 8, 128, 1, 1000)])
def test_append_q4_is_the_bf16_rows_quantised(rot, N, Hq, Hkv, D, blocks, rows):
    """Bit for bit: the codes of the row that the bf16 append writes, and its queries."""
    rng = np.random.default_rng(N)
    rot = dict(rot, rot_dim=min(rot["rot_dim"], D))
    q, k, v = fused_rows(rng, N, Hq, Hkv, D, torch.bfloat16)
    v[0, 0, 3] = float("nan")
    k[N - 1, 0, 1] = float("inf")
    k[N // 2, Hkv - 1] = 0.0
    pos = rng.integers(0, 131000, (3, N) if "sections" in rot else N)
    pos = dev(pos.astype(np.int32))
    slots = rng.permutation(blocks * rows)[:N].astype(np.int64)
    if N > 4:
        slots[3] = -1
    r = pv.Rotary(**rot)
    b16 = [torch.zeros((blocks, Hkv, rows, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = empty_cache((blocks, Hkv, rows), D, 0x5A)
    q1, q2 = (torch.full((N, Hq, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st = status_word()
    note(f"append q4 N{N} H{Hq}/{Hkv} D{D} {rot}")
    pv.rotary_append(q, k, v, pos, dev(slots), *b16, rotary=r, q_out=q1, status=st)
    pv.rotary_append_q4(q, k, v, pos, dev(slots), *cache, rotary=r, q_out=q2, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(q1.view(torch.int16), q2.view(torch.int16))
    live = np.zeros((blocks, rows), bool)
    ok = slots[slots >= 0]
    live[ok // rows, ok % rows] = True
    for x, c, e in ((b16[0], *cache[:2]), (b16[1], *cache[2:])):
        rc, re = Q.encode(x.double().cpu().numpy())
        c, e = host(c), host(e)
        m = np.broadcast_to(live[:, None], e.shape[:3])
        assert np.array_equal(c[m], Q.pack(rc)[m]) and np.array_equal(e[m], re[m])
        assert np.all(c[~m] == 0x5A) and np.all(e[~m] == 0x5A)


def test_rotary_flags_slots_past_the_cache():
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    rot, pos = pv.Rotary(rot_dim=64, base=1e4), i32([0, 0, 0])
    c = [torch.zeros((2, 2, 32, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q = torch.zeros_like(x)
    st = status_word()
    note("rotary: a slot past the cache")
    pv.rotary_append(x, x, x, pos, torch.tensor([63, 64, 1 << 40], device="cuda"), *c, rotary=rot, q_out=q, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == pv.PVLM_DEV_RANGE and q[0].all() and not q[1:].any()
    assert int((c[0] != 0).sum()) == 128 and c[1][1, :, 31].all()
    cache, st = empty_cache((2, 2, 32), 64), status_word()
    pv.rotary_append_q4(x, x, x, pos, torch.tensor([63, 64, 1 << 40], device="cuda"), *cache, rotary=rot, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == pv.PVLM_DEV_RANGE and int((cache[1] != 0).sum()) == 4


def test_rotary_in_place_and_on_another_stream():
    rng = np.random.default_rng(7)
    N, H, D = 70, 8, 128
    q, k, v = (dev(rows_like_a_models(rng, (N, h, D))).to(torch.bfloat16) for h in (H, 2, 2))
    rot, pos = pv.Rotary(rot_dim=64, base=1e6, layout="interleaved"), dev(np.arange(N, dtype=np.int32) * 31)
    slots = torch.arange(N, device="cuda")
    c = [torch.zeros((1, 2, 96, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    want = pv.rotary_append(q, k, v, pos, slots, *c, rotary=rot)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    mine = q.clone()
    torch.cuda.synchronize()
    note("rotary in place on a stream of its own")
    with torch.cuda.stream(s):
        got = pv.rotary_append(mine, k, v, pos, slots, *c, rotary=rot, q_out=mine)
    torch.cuda.synchronize()
    assert got is mine and torch.equal(mine, want)


def test_bindings_refuse_what_does_not_fit():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    z32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    rot, c = pv.Rotary(rot_dim=64, base=1e4), [bf(2, 2, 32, 64), bf(2, 2, 32, 64)]
    s = torch.zeros(5, dtype=torch.int64, device="cuda")
    good = dict(q=bf(5, 4, 64), k_new=bf(5, 2, 64), v_new=bf(5, 2, 64), pos=z32(5), slots=s, k_cache=c[0], v_cache=c[1],
                rotary=rot)

    def refuse(f, err=ValueError, **kw):
        with pytest.raises(err):
            f(**kw)
    for bad in (dict(q=bf(5, 4, 32)), dict(q=bf(4, 4, 64)), dict(q=bf(5, 4, 64).float()), dict(q=bf(5, 4, 128)[..., ::2]),
                dict(q=bf(4, 5, 64).transpose(0, 1)), dict(k_new=bf(5, 3, 64)), dict(v_new=bf(5, 2, 64).cpu()), dict(pos=z32(3, 5)),
                dict(pos=z32(5).long()), dict(slots=z32(5)), dict(slots=s[:4]), dict(k_cache=c[0][0]), dict(v_cache=bf(2, 2, 16, 64)),
                dict(k_cache=c[0].transpose(0, 1)), dict(q_out=bf(5, 4, 65))):
        refuse(pv.rotary_append, **{**good, **bad})
    refuse(pv.rotary_append, err=TypeError, **{**good, "rotary": None})
    refuse(pv.rotary_append, err=pv.PvlmError, **{**good, "rotary": pv.Rotary(rot_dim=128, base=1e4)})
    refuse(pv.rotary_append, **{**good, "rotary": pv.Rotary(rot_dim=64, base=1e4, sections=(8, 12, 12))})
    q4 = dict(zip(("k_codes", "k_exps", "v_codes", "v_exps"), empty_cache((2, 2, 32), 64)))
    rows = {k: v for k, v in good.items() if k not in ("k_cache", "v_cache")}
    refuse(pv.rotary_append_q4, **{**rows, **q4, "k_exps": q4["k_codes"]})
    refuse(pv.rotary_append_q4, **{**rows, **q4, "q": bf(5, 4, 64).float()})
    refuse(pv.rotary_append_q4, **{**rows, **q4, "k_codes": q4["k_codes"].float()})
    p = dict(length=z32(3), n_held=z32(3), page_table=z32(3, 4), free_pages=z32(9), n_free=z32(1), page_size=32)
    for bad in (dict(n_held=z32(2)), dict(page_table=z32(2, 4)), dict(free_pages=z32(3, 3)), dict(n_free=z32(2)),
                dict(length=z32(3).long()), dict(granted=z32(4)), dict(length=z32(3).cpu())):
        refuse(pv.pages_resize, **{**p, **bad})
    refuse(pv.pages_resize, err=pv.PvlmError, **{**p, "page_size": 33})
    m = dict(ctx_len=z32(3), n_new=z32(3), n_rows=9, page_size=32, n_pages=9, page_table=z32(3, 4))
    for bad in (dict(n_new=z32(2)), dict(page_table=z32(2, 4)), dict(page_table=None, n_pages=2), dict(ctx_len=z32(3, 1))):
        refuse(pv.slot_map, **{**m, **bad})
    refuse(pv.slot_map, err=pv.PvlmError, **{**m, "rows_per_seq": 2})
    refuse(pv.slot_map, err=pv.PvlmError, **{**m, "n_rows": 0})


# ---------------------------------------------------------------- together --
def test_a_paged_serving_step_as_a_graph():
    """What the calls are for: tables grown for a step's rows, their slots, the rotated rows appended to a paged 4-bit
    cache, verified, and the tables cut back to what was accepted, captured in one graph and replayed; every replay
    equals the same calls made one by one on a copy, and float64 attention over the values that the cache holds."""
    rng = np.random.default_rng(31)
    B, T, Hq, Hkv, D, P, max_pages, n_pages = 3, 5, 8, 2, 128, 32, 9, 40
    rot = pv.Rotary(rot_dim=64, base=1e6, layout="interleaved", scaling="yarn", factor=4.0, orig_ctx=4096.0, alpha=1.0, beta=32.0)
    ctx0 = [60, 0, 129]
    pool = Pool(B, P, max_pages, n_pages, seed=3)
    pool.resize(ctx0)
    held, table, free, n_free = pool.d
    cache = empty_cache((n_pages, Hkv, P), D)
    # the contexts, packed: a prefill's rows
    N0 = sum(ctx0)
    slots, pos, _, _ = pv.slot_map(i32([0] * B), i32(ctx0), N0, page_size=P, n_pages=n_pages, page_table=table)
    pv.rotary_append_q4(*fused_rows(rng, N0, Hq, Hkv, D, torch.bfloat16), pos, slots, *cache, rotary=rot)
    ctx, new = i32(ctx0), i32([5, 3, 5])
    q, k, v = fused_rows(rng, B * T, Hq, Hkv, D, torch.bfloat16)
    accepted = i32([2, 0, 5])
    want_len, qo = i32([0] * B), torch.zeros((B * T, Hq, D), dtype=torch.bfloat16, device="cuda")
    granted, kept = i32([9] * B), i32([9] * B)
    pv.default_status()

    def step(held, table, free, n_free, cache, ctx, q_out):
        torch.add(ctx, T, out=want_len)        # room for T rows a sequence: verify reads that many
        pv.pages_resize(want_len, held, table, free, n_free, page_size=P, granted=granted)
        slots, pos, seq, _ = pv.slot_map(ctx, new, B * T, page_size=P, n_pages=n_pages, page_table=table, rows_per_seq=T)
        pv.rotary_append_q4(q, k, v, pos, slots, *cache, rotary=rot, q_out=q_out)
        out, mass, lse = pv.verify_attn_q4_paged(q_out.view(B, T, Hq, D), *cache, table, ctx)
        ctx.add_(accepted).add_(1)
        pv.pages_resize(ctx, held, table, free, n_free, page_size=P, granted=kept)
        return slots, pos, seq, out, mass, lse
    copy = [t.clone() for t in (held, table, free, n_free, *cache, ctx)]
    warm = [t.clone() for t in copy]
    step(*warm[:4], warm[4:8], warm[8], qo.clone())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(held, table, free, n_free, cache, ctx, qo)
    qe = torch.zeros_like(qo)
    for i in range(4):
        note(f"paged serving step, replay {i}")
        c0 = ctx.tolist()
        g.replay()
        torch.cuda.synchronize()
        eager = step(*copy[:4], copy[4:8], copy[8], qe)
        torch.cuda.synchronize()
        # (rows of padding, which verify reads as queries and keys, are theirs as they were)
        for a, b in zip(got, eager):
            assert torch.equal(a, b)
        for a, b in zip((held, table, free, n_free, *cache, ctx), copy):
            assert torch.equal(a, b)
        # the table after the step holds what stays; the verify's pages are those of its slots
        top = free[:n_free.item()].tolist() + [x for row, h in zip(table.tolist(), held.tolist()) for x in row[:h]]
        assert sorted(top) == list(range(n_pages)) and held.tolist() == [-(-c // P) for c in ctx.tolist()]
        s = G.slot_map(c0, [5, 3, 5], B * T, P, None, T)
        assert got[1].tolist() == s[1] and got[2].tolist() == s[2]
    assert pv.synchronize() == 0
    # float64 over what the cache holds: one more step's verify, eager, over the rows of its table
    torch.add(ctx, T, out=want_len)
    pv.pages_resize(want_len, held, table, free, n_free, page_size=P)
    got = pv.verify_attn_q4_paged(qo.view(B, T, Hq, D), *cache, table, ctx)
    n = cap32(max(ctx.tolist()) + T)
    pad = []
    for t in cache:
        x = torch.zeros((B, Hkv, n, t.shape[-1]), dtype=torch.uint8, device="cuda")
        for b in range(B):
            for j in range(held[b].item()):
                x[b, :, j * P:(j + 1) * P] = t[table[b, j].item()][:, :n - j * P]
        pad.append(x)
    check_all((got[0], got[1][:, :n], got[2]), qo.view(B, T, Hq, D), pad, ctx.tolist())
