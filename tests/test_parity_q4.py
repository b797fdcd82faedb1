"""GPU parity of the 4-bit cache calls against plain float64 implementations.

* Rows written (append, quantise) are bit-exact: the format is one rounding of
  exactly scaled values (``oracle.quant4``).
* Verify is compared with float64 attention over the values that the rows stand
  for, within the bounds that ``test_parity_q8`` derives for the 8-bit call: they
  hold for exact operands in bf16, fp32 sums and a P rounded to bf16, whatever the
  rows are held in.
"""
import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
import workloads as W
from gpu_util import note
from oracle import quant4 as Q
from oracle.quant import bf16 as to_bf16
from test_parity_q8 import cap32, check, dev, paged, queries, reference, rows_like_a_models, status_word

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def host(t):
    return t.view(torch.uint8).cpu().numpy()


def values(codes, exps):
    """float64 values of a cache's tensors."""
    return dev(Q.decode(Q.unpack(host(codes)), host(exps)))


def to_cache(x):
    c, e = Q.encode(x)
    return dev(Q.pack(c)), dev(e)


def empty_cache(shape, D, fill=0):
    return [torch.full(shape + (w,), fill, dtype=torch.uint8, device="cuda") for w in (D // 2, D // 32) * 2]


def random_cache(rng, B, Hkv, rows, D, spread=0.0):
    side = []
    for _ in range(2):
        x = rows_like_a_models(rng, (B, Hkv, cap32(rows), D))
        if spread:
            x *= 2.0 ** rng.uniform(-spread, spread, x.shape[:-1] + (1,))
        side += to_cache(x)
    return side


# ------------------------------------------------------------------- rows --
SPECIAL = [0.0, -0.0, 7.0, 7.25, 1e-40, 3e38, -3e38, np.nan, np.inf, -np.inf, 2.0 ** -133, 5.0, 2.5]


def special_rows(rng, n, D):
    x = rows_like_a_models(rng, (n, D))
    x[0] = 0.0
    x[1] = 1e-39
    x[2] = 3.3e38 * np.sign(x[2])
    x[3, 3] = np.nan
    x[4, D - 1] = np.inf
    x[5] = np.nan
    x[6] = 2.0 ** rng.integers(-6, 3, D) * 1.25          # halfway values after scaling
    x[7] = 7.0
    x[8] = -5.0
    for i, s in enumerate(SPECIAL):
        x[9 + i, i] = s
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_quantise_special_rows_bit_exact(dtype, D):
    rng = np.random.default_rng(D)
    n = 77
    x, y = special_rows(rng, n, D), special_rows(rng, n, D)[::-1]
    cast = to_bf16 if dtype == "bf16" else (lambda a: a.astype(np.float32).astype(np.float64))
    with np.errstate(over="ignore"):
        x, y = cast(x), cast(y)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (dev(a.reshape(1, 1, n, D)).to(tdt) for a in (x, y))
    cache = empty_cache((1, 1, cap32(n)), D, 0xAB)
    note(f"quantise q4 special rows {dtype} D={D}")
    st = status_word()
    pv.quantize_kv_q4(k, v, i32([n]), *cache, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for a, c, e in ((x, *cache[:2]), (y, *cache[2:])):
        rc, re = Q.encode(a)
        assert np.array_equal(host(e)[0, 0, :n], re)
        got = Q.unpack(host(c)[0, 0, :n])
        off = np.argwhere(got != rc)
        assert not len(off), [(tuple(i), a[tuple(i)], got[tuple(i)], rc[tuple(i)]) for i in off[:4]]
        assert np.all(host(c)[0, 0, n:] == 0xAB) and np.all(host(e)[0, 0, n:] == 0xAB)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L,B,Hkv,D,lens,src_cap,P", [
    (1, 1, 1, 64, [1], 1, 0), (3, 2, 4, 128, [70, 0], 71, 0), (2, 3, 2, 64, [5, 200, 64], 200, 32),
    (28, 1, 4, 128, [301], 333, 64), (1, 4, 8, 128, [33, 1, 512, 31], 600, 256),
])
def test_quantise_stacked(L, B, Hkv, D, lens, src_cap, P, dtype):
    rng = np.random.default_rng(L + B + D)
    cast = to_bf16 if dtype is torch.bfloat16 else (lambda a: a.astype(np.float32).astype(np.float64))
    x = [cast(rows_like_a_models(rng, (L, B, Hkv, src_cap, D))) for _ in range(2)]
    k, v = (dev(a).to(dtype) for a in x)
    note(f"quantise q4 stacked L{L} B{B} H{Hkv} D{D} lens{lens} P{P}")
    st = status_word()
    if P:
        table, n_pages = W.page_table(np.array(lens), P, seed=4)
        cache = empty_cache((L, n_pages, Hkv, P), D, 0xC3)
        pv.quantize_kv_q4_paged(k, v, i32(lens), *cache, dev(table), status=st)
    else:
        cache = empty_cache((L, B, Hkv, cap32(max(lens))), D, 0xC3)
        pv.quantize_kv_q4(k, v, i32(lens), *cache, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for a, c, e in ((x[0], host(cache[0]), host(cache[1])), (x[1], host(cache[2]), host(cache[3]))):
        rc, re = Q.encode(a)
        rc = Q.pack(rc)
        seen = np.zeros(e.shape[:-1], bool)
        for b, n in enumerate(lens):
            for i in range(n):
                at = (slice(None), table[b, i // P], slice(None), i % P) if P else (slice(None), b, slice(None), i)
                assert np.array_equal(c[at], rc[:, b, :, i]) and np.array_equal(e[at], re[:, b, :, i])
                seen[at] = True
        assert np.all(c[~seen] == 0xC3) and np.all(e[~seen] == 0xC3)


def test_quantise_flags_lengths_and_pages():
    k = torch.randn((1, 2, 40, 64), device="cuda")
    cache = empty_cache((1, 2, 32), 64)
    for n, flagged in ((41, True), (33, True), (-1, True), (32, False)):
        st = status_word()
        note(f"quantise q4 length {n} of 40 rows into 32")
        pv.quantize_kv_q4(k, k, i32([n]), *cache, status=st)
        assert bool(int(st.item()) & pv.PVLM_DEV_RANGE) == flagged
    pool = empty_cache((3, 2, 32), 64)
    st = status_word()
    pv.quantize_kv_q4_paged(k, k, i32([40]), *pool, i32([[1, 9]]), status=st)
    assert int(st.item()) & pv.PVLM_DEV_RANGE
    assert pool[1][1].any() and not pool[1][[0, 2]].any()


# ----------------------------------------------------------------- verify --
def run_verify(q, cache, ctx, scale=None, P=0, seed=0, max_ctx=None, want_mass=True, garbage=True):
    """The call on a padded and (P) paged cache whose unwritten rows hold full codes of exponent 255 (NaN)."""
    B, T, Hq, D = q.shape
    cache = [c.clone() for c in cache]
    if garbage:
        for b, c in enumerate(ctx):
            for t in cache:
                t[b, :, c + T:] = 0xff
    st = status_word()
    kw = dict(scale=scale, status=st, want_mass=want_mass)
    got = pv.verify_attn_q4(q, *cache, i32(ctx), max_ctx=max_ctx, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    if P:
        table, n_pages = W.page_table(np.array(ctx) + T, P, seed=seed)
        pools = [paged(t, table, n_pages, P, 0xff) for t in cache]
        # an equal max_ctx gives the padded call's plan, so the results are the same bits
        mc = max(ctx) if max_ctx is None else max_ctx
        got = pv.verify_attn_q4(q, *cache, i32(ctx), max_ctx=mc, **kw)
        pg = pv.verify_attn_q4_paged(q, *pools, dev(table), i32(ctx), max_ctx=mc, **kw)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        n = cache[0].shape[2]
        assert torch.equal(got[0].view(torch.int16), pg[0].view(torch.int16))
        assert torch.equal(got[2].view(torch.int32), pg[2].view(torch.int32))
        if want_mass:
            m = min(n, pg[1].shape[1])
            assert torch.equal(got[1][:, :m].view(torch.int32), pg[1][:, :m].view(torch.int32))
            assert not pg[1][:, m:].any()
    return got


def check_all(got, q, cache, ctx, scale=None):
    out, mass, lse = got
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, scale)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")
    if mass is not None:
        check(mass[:, :rm.shape[1]], rm, bm, "mass")
        for b, c in enumerate(ctx):
            assert not mass[b, c + q.shape[1]:].any()


VERIFIES = [
    # B, T, Hq, Hkv, D, ctx, P
    (1, 1, 1, 1, 64, [0], 0),                       # one token sees itself
    (1, 1, 7, 1, 128, [0], 32),
    (1, 4, 2, 2, 64, [1], 0),
    (3, 5, 8, 2, 128, [300, 517, 31], 32),          # ragged, pages that end inside a tile
    (2, 9, 64, 8, 128, [1111, 700], 64),            # 5 row tiles
    (2, 2, 8, 2, 64, [190, 1000], 32),
    (1, 32, 16, 2, 128, [700], 256),                # T = 32, 16 tiles over two workgroups
    (1, 32, 20, 1, 64, [333], 0),                   # 640 rows per KV head: 40 tiles
    (1, 3, 8, 8, 128, [9000], 32),
    (4, 9, 28, 4, 128, [100, 900, 3, 1500], 32),
    (1, 17, 64, 8, 128, [5000], 32),                # 9 row tiles
    (16, 1, 28, 4, 128, [97 * i for i in range(16)], 64),   # a decode batch, one sequence empty but for its token
    (1, 1, 8, 8, 64, [63], 0), (1, 1, 8, 8, 64, [62], 0), (1, 1, 8, 8, 64, [64], 0),
    (1, 5, 4, 1, 64, [255], 0), (1, 5, 4, 1, 64, [252], 0), (1, 6, 4, 4, 128, [122], 0),
    (1, 11, 6, 1, 128, [777], 0), (1, 15, 6, 1, 64, [1000], 32),      # 5 and 6 tiles
    (1, 16, 7, 1, 128, [500], 0), (1, 16, 8, 1, 64, [600], 0),        # 7 and 8 tiles
    (1, 9, 5, 1, 128, [400], 0), (1, 9, 7, 1, 64, [400], 32),         # 3 and 4 tiles
    (2, 3, 3, 3, 128, [2000, 50], 32), (1, 2, 30, 6, 64, [3333], 0),  # KV heads that are no power of two
]


@pytest.mark.parametrize("case", VERIFIES, ids=lambda c: f"B{c[0]}T{c[1]}H{c[2]}/{c[3]}D{c[4]}c{c[5][0]}P{c[6]}")
def test_verify_shapes(case):
    B, T, Hq, Hkv, D, ctx, P = case
    rng = np.random.default_rng(sum(ctx) + 7 * T + D)
    q, cache = queries(rng, B, T, Hq, D), random_cache(rng, B, Hkv, max(ctx) + T, D)
    note(f"verify q4 {case}")
    got = run_verify(q, cache, ctx, P=P, seed=B)
    check_all(got, q, cache, ctx)
    # without the mass, and with the shorter plan of the true longest context
    out, none, lse = run_verify(q, cache, ctx, max_ctx=max(ctx), want_mass=False)
    assert none is None
    check_all((out, None, lse), q, cache, ctx)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(3, 4), (4, 7), (9, 5), (9, 7), (10, 8), (12, 8), (16, 7), (32, 4), (17, 8), (32, 5),
                                 (32, 6)])
def test_verify_every_number_of_row_tiles(T, G, D):
    """1 to 10 tiles of 16 rows, and 12; pages of one unit."""
    rng = np.random.default_rng(T * G + D)
    ctx = [261, 1337]
    q, cache = queries(rng, 2, T, 2 * G, D), random_cache(rng, 2, 2, max(ctx) + T, D)
    note(f"verify q4 tiles T={T} G={G} D={D}")
    check_all(run_verify(q, cache, ctx, P=32, seed=T), q, cache, ctx)


@pytest.mark.parametrize("B", [64, 65, 200])
def test_verify_many_sequences(B):
    """More sequences than a wave has lanes; lengths from 0 on, some workgroups with pieces of several sequences."""
    rng = np.random.default_rng(B)
    T, Hq, Hkv, D = 2, 6, 2, 64
    ctx = [int(x) for x in rng.integers(0, 400, B)]
    ctx[0], ctx[B // 2], ctx[B - 1] = 0, 30, 1
    q, cache = queries(rng, B, T, Hq, D), random_cache(rng, B, Hkv, max(ctx) + T, D)
    note(f"verify q4 {B} sequences")
    check_all(run_verify(q, cache, ctx, P=32, seed=B), q, cache, ctx)


def test_verify_long_contexts():
    """131K rows, 136 query rows a KV head; and a decode step over the same cache."""
    rng = np.random.default_rng(3)
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    B, T, Hq, Hkv, D, ctx = 1, 17, 16, 2, 128, 131072 - 17
    x = [torch.randn((B, Hkv, 131072, D), device="cuda", generator=g) for _ in range(2)]
    cache = empty_cache((B, Hkv, 131072), D)
    pv.quantize_kv_q4(*x, i32([131072]), *cache)
    q = queries(rng, B, T, Hq, D)
    note("verify q4 131K, T = 17")
    check_all(run_verify(q, cache, [ctx]), q, cache, [ctx])
    one = q[:, :1].contiguous()
    note("verify q4 131K, T = 1")
    check_all(run_verify(one, cache, [131071], want_mass=False), one, cache, [131071])


def test_verify_offsets_past_32_bits():
    """A pool of more than 2^32 bytes of codes: the sequence's pages are its last ones."""
    P, Hkv, D, n_pages = 1024, 8, 128, 8300      # 4.35 GB of codes a side
    rng = np.random.default_rng(5)
    ctx, T, Hq = [4000], 3, 16
    side = random_cache(rng, 1, Hkv, 4096, D)
    pools = [torch.zeros((n_pages, Hkv, P) + t.shape[3:], dtype=torch.uint8, device="cuda") for t in side]
    table = i32([[n_pages - 1 - 2 * i for i in range(4)]])
    for i in range(4):
        for t, p in zip(side, pools):
            p[int(table[0, i])] = t[0, :, i * P:(i + 1) * P]
    q = queries(rng, 1, T, Hq, D)
    note("verify q4 over a pool past 4 GB")
    want = pv.verify_attn_q4(q, *side, i32(ctx), max_ctx=ctx[0])
    got = pv.verify_attn_q4_paged(q, *pools, table, i32(ctx), max_ctx=ctx[0])
    torch.cuda.synchronize()
    assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[2], want[2])
    assert torch.equal(got[1], want[1][:, :4096])
    kn = queries(rng, 1, T, Hkv, D)[0]
    rot = pv.Rotary(rot_dim=D, base=1e6)
    slots, pos, _, _ = pv.slot_map(i32(ctx), i32([T]), T, page_size=P, n_pages=n_pages, page_table=table)
    pv.rotary_append_q4(q[0], kn, kn, pos, slots, *pools, rotary=rot)
    pv.rotary_append_q4(q[0], kn, kn, pos, torch.arange(T, device="cuda") + ctx[0], *side, rotary=rot)
    page = int(table[0, 3])
    for p, t in zip(pools, side):
        assert torch.equal(p[page, :, 4000 - 3 * P:4003 - 3 * P], t[0, :, 4000:4003])
    e = torch.zeros((1, 0), dtype=torch.int32, device="cuda")
    back = pv.gather_kv_q4_paged(*pools, table, e, i32([0]), i32([4000]), i32([3]), 32)
    assert all(torch.equal(b[0, :, :3], t[0, :, 4000:4003]) for b, t in zip(back, side))


@pytest.mark.parametrize("D", [64, 128])
def test_verify_wide_ranges(D):
    """Values whose units differ by 2^24, a key that dwarfs the others (a sink), queries with one large channel."""
    rng = np.random.default_rng(D + 1)
    B, T, Hq, Hkv, ctx = 1, 6, 8, 2, [1500]
    cache = random_cache(rng, B, Hkv, ctx[0] + T, D, spread=12.0)
    ks = random_cache(rng, B, Hkv, ctx[0] + T, D)[:2]
    q = queries(rng, B, T, Hq, D)
    q[..., 5] *= 64.0
    sink = q[0].double().mean(dim=(0, 1))
    x = values(*ks)[0].cpu().numpy()
    x[:, 0] = (sink / sink.norm() * 20).cpu().numpy()
    c, e = to_cache(x)
    ks[0][0], ks[1][0] = c, e
    cache = [*ks, *cache[2:]]
    note(f"verify q4 wide ranges D={D}")
    check_all(run_verify(q, cache, ctx, P=32), q, cache, ctx)


def test_verify_zero_and_extreme_queries():
    rng = np.random.default_rng(12)
    ctx, T, D = [200], 4, 128
    cache = random_cache(rng, 1, 1, ctx[0] + T, D)
    q = queries(rng, 1, T, 4, D)
    q[0, 0] = 0.0                       # the mean of the values
    q[0, 1] *= 2.0 ** -40
    q[0, 2, 0] *= 2.0 ** 20             # one key takes all
    q[0, 3, 0, 1:] *= 2.0 ** -20        # one channel holds all but 2^-20
    note("verify q4 zero, tiny and huge queries")
    out, mass, lse = run_verify(q, cache, ctx)
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, D ** -0.5)
    keep = torch.ones((1, T, 4), dtype=torch.bool, device="cuda")
    keep[0, 2, 0] = False               # (a bound of scores this large says nothing)
    check(out[keep], ro[keep], bo[keep], "out")
    check(lse.transpose(1, 2)[keep], rl.transpose(1, 2)[keep], bl.transpose(1, 2)[keep], "lse")
    top = (q[0, 2, 0].double() @ values(*cache[:2])[0, 0, :ctx[0] + 3].t()).argmax()
    # (P of that key is 1 but for terms under 2^-60, and the result is its value, a bf16 number)
    assert torch.equal(out[0, 2, 0].double(), values(*cache[2:])[0, 0, top])


@pytest.mark.parametrize("ctx,T,D", [([190], 6, 128), ([31], 8, 64), ([700], 32, 128)])
def test_verify_nan_reaches_only_the_rows_that_see_it(ctx, T, D):
    """An exponent of 255 is 32 NaN, in a K or V row of the verify block (rows behind it see it) or of the context."""
    rng = np.random.default_rng(6)
    Hq, Hkv = 8, 2
    cache = random_cache(rng, 1, Hkv, ctx[0] + T, D)
    q = queries(rng, 1, T, Hq, D)
    clean, _, clse = run_verify(q, cache, ctx, P=32)
    bad = [t.clone() for t in cache]
    bad[3][0, 1, ctx[0] + 3, 1] = 255        # V: columns 32 .. 63 of the second KV head, seen by t >= 3
    bad[1][0, 0, ctx[0] + 5, 0] = 255        # K: the first KV head, seen by t >= 5
    note("verify q4 NaN in the draft's rows")
    out, mass, lse = run_verify(q, bad, ctx, P=32)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[0, 3:, 4:, 32:64] = True
    want[0, 5:, :4] = True
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(torch.isnan(lse[0]), want[0, :, :, 0].t())
    assert torch.equal(out[~want].view(torch.int16), clean[~want].view(torch.int16))
    # the mass of what a row of NaN sees is NaN: everything up to the last row's own token
    assert torch.isnan(mass[0, :ctx[0] + T]).all() and not mass[0, ctx[0] + T:].any()
    bad = [t.clone() for t in cache]
    bad[3][0, 0, 5, 1] = 255                 # V in the context: every row of the head
    q2 = q.clone()
    q2[0, 2, 6, 9] = float("inf")            # a query: its own row
    out, mass, lse = run_verify(q2, bad, ctx)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[0, :, :4, 32:64] = True
    want[0, 2, 6] = True
    assert torch.equal(torch.isnan(out), want)


@pytest.mark.parametrize("T,D,ctx", [(8, 64, [63, 0]), (32, 128, [90, 33]), (17, 128, [5000, 40])])
def test_nan_in_every_draft_row_reaches_the_rows_that_see_it(T, D, ctx):
    rng = np.random.default_rng(T)
    cache = random_cache(rng, 2, 2, max(ctx) + T, D)
    q = queries(rng, 2, T, 4, D)
    for b, c in enumerate(ctx):
        for t in range(T):
            cache[3][b, 1, c + t, t % (D // 32)] = 255
    note(f"verify q4 NaN in {T} rows")
    out, _, lse = run_verify(q, cache, ctx, P=32, seed=3)
    want = torch.zeros_like(out, dtype=torch.bool)
    for t in range(T):
        k = t % (D // 32)
        want[:, t:, 2:, 32 * k:32 * k + 32] = True
    assert torch.equal(torch.isnan(out), want) and not torch.isnan(lse).any()


def test_verify_context_out_of_range_is_clamped_and_flagged():
    rng = np.random.default_rng(9)
    T, Hq, Hkv, D = 3, 4, 2, 64
    cache = random_cache(rng, 2, Hkv, 128, D)
    q = queries(rng, 2, T, Hq, D)
    st = status_word()
    note("verify q4 contexts outside [0, max_ctx]")
    got = pv.verify_attn_q4(q, *cache, i32([-4, 5000]), max_ctx=100, status=st)
    want = pv.verify_attn_q4(q, *cache, i32([0, 100]), max_ctx=100)
    torch.cuda.synchronize()
    assert int(st.item()) & pv.PVLM_DEV_RANGE
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_verify_bad_page_entry_is_flagged_and_stays_in_the_pool():
    rng = np.random.default_rng(10)
    ctx, T, D = [300, 200], 3, 128
    cache = random_cache(rng, 2, 2, 303, D)
    table, n_pages = W.page_table(np.array(ctx) + T, 32, seed=3)
    pools = [paged(t, table, n_pages, 32, 0x38) for t in cache]
    q = queries(rng, 2, T, 8, D)
    for entry in (n_pages + 7, -1):
        table[1, 2] = entry
        for mass in (True, False):
            st = status_word()
            note(f"verify q4 page entry {entry}, pool of {n_pages}, mass {mass}")
            pv.verify_attn_q4_paged(q, *pools, dev(table), i32(ctx), want_mass=mass, status=st)
            torch.cuda.synchronize()
            assert int(st.item()) & pv.PVLM_DEV_RANGE


def test_verify_is_the_same_each_time_on_any_stream_and_budget():
    rng = np.random.default_rng(14)
    ctx, T, Hq, Hkv, D = [3001], 9, 64, 8, 128
    cache = random_cache(rng, 1, Hkv, ctx[0] + T, D)
    q = queries(rng, 1, T, Hq, D)
    first = pv.verify_attn_q4(q, *cache, i32(ctx))
    n = i32(ctx)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, pv.verify_attn_q4(q, *cache, n)))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    note("verify q4 on two streams at once")
    outs = []
    for _ in range(4):
        for s in (s1, s2):
            with torch.cuda.stream(s):
                outs.append(pv.verify_attn_q4(q, *cache, n))
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(first, o))
    for cus in (8, 32):
        note(f"verify q4 on a stream of {cus} compute units")
        pv.set_stream_cu_budget(s1, cus)
        try:
            with torch.cuda.stream(s1):
                got = pv.verify_attn_q4(q, *cache, n)
            torch.cuda.synchronize()
        finally:
            pv.set_stream_cu_budget(s1, 0)
        check_all(got, q, cache, ctx)


def test_workspace_is_checked_and_holds_nothing_between_calls():
    """A workspace one byte short is refused; one full of NaN serves; the region of captured bf16 calls is left."""
    rng = np.random.default_rng(15)
    ctx, T, Hq, Hkv, D = [900], 5, 8, 2, 128
    cache = random_cache(rng, 1, Hkv, ctx[0] + T, D)
    n_cap = cache[0].shape[2]
    q = queries(rng, 1, T, Hq, D)
    need = pv.verify_attn_q4_workspace_size(1, T, Hq, Hkv, D, n_cap, n_cap - T)

    class Buffer:
        def __init__(self, extra, fill):
            self.extra, self.fill = extra, fill

        def get(self, n):
            assert n == need
            self.buf = torch.full((n + self.extra + 64,), self.fill, dtype=torch.uint8, device="cuda")
            return self.buf[:n + self.extra]
    with pytest.raises(pv.PvlmError) as err:
        pv.verify_attn_q4(q, *cache, i32(ctx), ws=Buffer(-1, 0))
    assert err.value.status == 4
    want = pv.verify_attn_q4(q, *cache, i32(ctx))
    full = Buffer(0, 0xff)
    got = pv.verify_attn_q4(q, *cache, i32(ctx), ws=full)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool((full.buf[need:] == 0xff).all()) and bool((full.buf[:1 << 20] == 0xff).all())


def test_graphs_of_one_capture_stream_replay_together():
    """Captured calls without a workspace of their own have one of their graph's: two graphs replayed at once on two
    streams, among eager calls."""
    rng = np.random.default_rng(21)
    shapes = [([700, 90], 5, 8, 2, 128), ([3000], 17, 16, 2, 64)]
    work = [(queries(rng, len(c), T, Hq, D), random_cache(rng, len(c), Hkv, max(c) + T, D), i32(c))
            for c, T, Hq, Hkv, D in shapes]
    want = [pv.verify_attn_q4(q, *c, n) for q, c, n in work]
    pv.default_status()
    torch.cuda.synchronize()
    graphs, got = [], []
    for q, c, n in work:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(pv.verify_attn_q4(q, *c, n))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    note("verify q4: two graphs on two streams")
    for _ in range(4):
        for o in got:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = [pv.verify_attn_q4(q, *c, n) for q, c, n in work]
        torch.cuda.synchronize()
        for o, e, w in zip(got, eager, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w)) and all(torch.equal(a, b) for a, b in zip(e, w))
    assert pv.synchronize() == 0


def test_verify_small_probabilities_beside_a_large_one():
    """One key of score 18 (the row holds it exactly), 40000 of score 0, each a small part of the last place of the large
    one.  Scores are exact (one channel), so the log-sum-exp is off by five roundings of its size and the logarithm's
    2^-20."""
    B, Hkv, D, n = 4, 8, 64, 40000
    x = np.zeros((B, Hkv, cap32(n + 1), D))
    x[:, :, 37, 0] = 16.0
    cache = [*to_cache(x), *to_cache(np.ones_like(x))]
    q = torch.zeros((B, 1, Hkv, D), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.125
    note("verify q4 one large probability among small ones")
    out, mass, lse = run_verify(q, cache, [n] * B, scale=1.0, garbage=False)
    want = np.logaddexp(18.0, np.log(n))
    assert (lse.double() - want).abs().max().item() <= 5 * 18.0 * 2.0 ** -24 + 2.0 ** -20
    assert torch.equal(out, torch.ones_like(out))
    p = np.exp(-want)
    assert (mass[:, 1000:n].double() / (Hkv * p) - 1).abs().max().item() <= 2.0 ** -16


def test_verify_small_probabilities_in_long_shares():
    """Sequences of 100000 tokens on a compute unit each, one score 0, all others -28 (in steps of log 2; every score is
    exact).  A lane sums 3125 tokens, eight at a time: 2^-25 of the large one, half of what moves it.  It may lose those
    of the first 16 units (2^-21), round once for each further 16 (25 half places of 2^-23) and in the joins (10 more),
    and the logarithm is off by 2^-20; all of them lost would be 1.2e-5."""
    B, D, n, cus = 8, 64, 100000, 8
    cache = empty_cache((B, 1, cap32(n + 1)), D)
    cache[1][:] = cache[3][:] = 127
    cache[0][..., :14] = 0xAA                       # -1 in 28 channels
    cache[0][:, :, 37] = 0
    cache[2][:] = 0x22                              # values 1
    q = torch.ones((B, 1, 1, D), dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    note("verify q4 small probabilities in long shares")
    pv.set_stream_cu_budget(stream, cus)
    try:
        with torch.cuda.stream(stream):
            out, mass, lse = pv.verify_attn_q4(q, *cache, i32([n] * B), scale=float(np.log(2.0)))
        torch.cuda.synchronize()
    finally:
        pv.set_stream_cu_budget(stream, 0)
    z = 1 + n * 2.0 ** -28
    assert (lse.double() - np.log(z)).abs().max().item() <= 2.0 ** -21 + 35 * 2.0 ** -24 + 2.0 ** -20
    assert torch.equal(out, torch.ones_like(out))
    assert (mass[:, 1000:n].double() * 2.0 ** 28 * z - 1).abs().max().item() <= 2.0 ** -16


def test_every_token_counts_once():
    """Equal scores: the mass of every visible token is Hq * T / n to 2^-16, at lengths around the units and shares."""
    for B, T, Hq, Hkv, D, ctx in [(1, 1, 8, 2, 64, [20000]), (2, 4, 8, 8, 128, [8190, 4097]), (3, 2, 4, 1, 128, [65, 31, 0])]:
        cache = empty_cache((B, Hkv, cap32(max(ctx) + T)), D)
        for e in (1, 3):
            cache[e][:] = 127
        cache[2][:] = 0x22                     # values 1
        q = torch.ones((B, T, Hq, D), dtype=torch.bfloat16, device="cuda")
        note(f"verify q4 equal scores {ctx}")
        out, mass, lse = run_verify(q, cache, ctx, P=32)
        assert torch.equal(out, torch.ones_like(out))
        for b, c in enumerate(ctx):
            n = torch.arange(c + 1, c + T + 1, dtype=torch.float64, device="cuda")
            assert (lse[b].double() - n.log()).abs().max() <= 2.0 ** -20 + 2.0 ** -23 * 12
            want = torch.stack([(torch.arange(c + T, device="cuda") <= c + t).double() / n[t] for t in range(T)]).sum(0) * Hq
            assert (mass[b, :c + T].double() / want - 1).abs().max() <= 2.0 ** -16


# ----------------------------------------------------------------- gather --
@pytest.mark.parametrize("dtype", [torch.uint8, torch.float4_e2m1fn_x2, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("P,D", [(0, 128), (64, 64), (32, 128)])
def test_gather(dtype, P, D):
    L, B, Hkv = 3, 3, 4
    rng = np.random.default_rng(11 + D)
    rows = np.array([1500, 64, 700])
    n_cap = cap32(int(rows.max()))
    codes = [rng.integers(0, 256, (L, B, Hkv, n_cap, D // 2)).astype(np.uint8) for _ in range(2)]
    exps = [rng.integers(0, 256, (L, B, Hkv, n_cap, D // 32)).astype(np.uint8) for _ in range(2)]
    exps[0][:, 0, 0, :40] = 1
    K = np.array([300, 0, 500], np.int32)
    k_cap = 520
    idx = np.full((B, k_cap), -1, np.int32)
    for b in range(B):
        idx[b, :K[b]] = np.sort(rng.choice(rows[b] - 40, size=K[b], replace=False))
    idx[0, 5] = idx[0, 4]                         # the same row twice
    tb, tl = (rows - 40).astype(np.int32), np.full(B, 40, np.int32)
    dst_cap = 576
    sides = [codes[0], exps[0], codes[1], exps[1]]
    if P:
        table, n_pages = W.page_table(rows, P, seed=12)
        sides = [np.stack([W.to_pages(a[l], table, n_pages, P) for l in range(L)]) for a in sides]
    cache = [dev(a) for a in sides]
    sel = [dev(a) for a in (idx, K, tb, tl)]
    note(f"gather q4 {dtype} P={P} D={D}")
    st = status_word()
    q4 = dtype in (torch.uint8, torch.float4_e2m1fn_x2)

    def call(dst=None):
        if P:
            return pv.gather_kv_q4_paged(*cache, dev(table), *sel, dst_cap, dtype=dtype, dst=dst, status=st)
        return pv.gather_kv_q4(*cache, *sel, dst_cap, dtype=dtype, dst=dst, status=st)
    got = call()
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    shape = (L, B, Hkv, dst_cap)
    old = empty_cache(shape, D, 0x77) if q4 else [torch.full(shape + (D,), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    kept = call(old)
    torch.cuda.synchronize()
    for side in range(2):
        want_c, want_e = np.zeros(shape + (D // 2,), np.uint8), np.zeros(shape + (D // 32,), np.uint8)
        live = np.zeros(shape, bool)
        for b in range(B):
            src = np.concatenate([idx[b, :K[b]], tb[b] + np.arange(tl[b])])
            want_c[:, b, :, :len(src)] = codes[side][:, b][:, :, src]
            want_e[:, b, :, :len(src)] = exps[side][:, b][:, :, src]
            live[:, b, :, :len(src)] = True
        if q4:
            assert np.array_equal(host(got[2 * side]), want_c) and np.array_equal(host(got[2 * side + 1]), want_e)
            assert np.array_equal(host(kept[2 * side])[live], want_c[live])
            assert np.all(host(kept[2 * side])[~live] == 0x77) and np.all(host(kept[2 * side + 1])[~live] == 0x77)
        else:
            with np.errstate(over="ignore"):
                v = torch.from_numpy(Q.decode(Q.unpack(want_c), want_e)).to(torch.float32).to(dtype).cuda()
            v[~dev(live)] = 0.0
            assert torch.equal(torch.isnan(got[side]), torch.isnan(v))
            assert torch.equal(got[side].nan_to_num(nan=1.5), v.nan_to_num(nan=1.5))
            live = dev(live)
            assert torch.equal(kept[side][live].nan_to_num(), got[side][live].nan_to_num())
            assert bool((kept[side][~live] == 7.0).all())


def test_gather_flags_what_is_out_of_range():
    cache = [torch.randint(1, 100, s, dtype=torch.uint8, device="cuda") for s in ((1, 2, 64, 32), (1, 2, 64, 2)) * 2]

    def call(idx, k, tb, tl, cap=32):
        st = status_word()
        r = pv.gather_kv_q4(*cache, i32([idx]), i32([k]), i32([tb]), i32([tl]), cap, status=st)
        return bool(int(st.item()) & pv.PVLM_DEV_RANGE), r
    note("gather q4 indices, counts and tails out of range")
    assert not call([1, 2], 2, 60, 4)[0]
    bad, r = call([1, 64], 2, 60, 4)
    assert bad and not r[1][0, :, 1].any() and r[1][0, :, [0, 2, 3, 4, 5]].all()
    for args in (([1, -1], 2, 60, 4), ([1, 2], 3, 60, 4), ([1, 2], -1, 60, 4), ([1, 2], 2, 65, 0),
                 ([1, 2], 2, 60, 5), ([1, 2], 2, 30, 31), ([1, 2], 2, 30, -1)):
        assert call(*args)[0], args
    pool = [torch.randint(1, 100, s, dtype=torch.uint8, device="cuda") for s in ((2, 2, 32, 32), (2, 2, 32, 2)) * 2]
    st = status_word()
    r = pv.gather_kv_q4_paged(*pool, i32([[1, 2]]), i32([[3, 40]]), i32([2]), i32([5]), i32([1]), 32, status=st)
    assert int(st.item()) & pv.PVLM_DEV_RANGE
    assert torch.equal(r[1][0, :, [0, 2]], pool[1][1, :, [3, 5]]) and not r[1][0, :, 1].any()


# --------------------------------------------------------------- refusals --
def test_bindings_refuse_what_does_not_fit():
    B, T, Hq, Hkv, D, n = 2, 3, 4, 2, 64, 64
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    z32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    cache = empty_cache((B, Hkv, n), D)
    q, kn = bf(B, T, Hq, D), bf(B, Hkv, 10, D)

    def refuse(f, *a, err=ValueError, **kw):
        with pytest.raises(err):
            f(*a, **kw)
    short = [cache[0], cache[1][:, :, :32].contiguous(), *cache[2:]]
    strided = [cache[0].transpose(1, 2).contiguous().transpose(1, 2), *cache[1:]]
    wrong = [cache[0].to(torch.int32), *cache[1:]]
    host_ = [cache[0].cpu(), *cache[1:]]
    for c in (short, strided, wrong, host_, empty_cache((B, Hkv, n), 32), empty_cache((B, Hkv, n), 96)):
        refuse(pv.verify_attn_q4, q, *c, z32(B))
        refuse(pv.quantize_kv_q4, kn, kn, z32(B), *c)
        refuse(pv.gather_kv_q4, *c, z32(B, 4), z32(B), z32(B), z32(B), 32)
    refuse(pv.verify_attn_q4, q.float(), *cache, z32(B))
    refuse(pv.verify_attn_q4, q[:1], *cache, z32(1))
    refuse(pv.verify_attn_q4, q, *cache, z32(B + 1))
    refuse(pv.verify_attn_q4, q, *cache, z32(B), out=bf(B, T, Hq, D + 1))
    refuse(pv.verify_attn_q4, q, *cache, z32(B), mass=torch.zeros((B, n + 1), device="cuda"))
    refuse(pv.verify_attn_q4, q, *cache, z32(B), lse=torch.zeros((B, T, Hq), device="cuda"))
    refuse(pv.verify_attn_q4, q, *cache, z32(B), max_ctx=n, err=pv.PvlmError)
    refuse(pv.verify_attn_q4_paged, q, *cache, None, z32(B), err=TypeError)
    refuse(pv.verify_attn_q4_paged, q, *cache, z32(1, 4), z32(B))
    refuse(pv.quantize_kv_q4, kn[None], kn[None], z32(B), *cache)
    refuse(pv.quantize_kv_q4, kn.half(), kn.half(), z32(B), *cache)
    refuse(pv.quantize_kv_q4_paged, kn, kn, z32(B), *cache, None, err=TypeError)
    refuse(pv.gather_kv_q4, *cache, z32(B, 4), z32(B), z32(B), z32(B), 32, dtype=torch.float16)
    refuse(pv.gather_kv_q4, *cache, z32(B, 4), z32(B), z32(B), z32(B), 33, err=pv.PvlmError)
    refuse(pv.gather_kv_q4, *cache, z32(B, 4), z32(B), z32(B), z32(B), 32, dst=cache)
    refuse(pv.gather_kv_q4, *cache, z32(B, 4), z32(B + 1), z32(B), z32(B), 32)
    refuse(pv.gather_kv_q4_paged, *cache, None, z32(B, 4), z32(B), z32(B), z32(B), 32, err=TypeError)
    off = torch.zeros(B * Hkv * n * D // 2 + 1, dtype=torch.uint8, device="cuda")[1:].view(B, Hkv, n, D // 2)
    refuse(pv.verify_attn_q4, q, off, *cache[1:], z32(B), err=pv.PvlmError)      # codes not 16-byte aligned
