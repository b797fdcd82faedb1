"""GPU parity of the 8-bit cache calls against plain float64 implementations.

* Rows written (append, quantise) are bit-exact: the format is one rounding of
  exactly scaled values (``oracle.quant``).
* Verify is compared with float64 attention over the values that the rows stand
  for.  Its bound, per result, from the arithmetic the call documents:
  - a score is off by at most  ds = scale * sum_d |q_d k_d| * (D + 4) 2^-24: exact
    products, fp32 sums of D of them;
  - a probability is off, relative to itself, by at most
    dp = 2 (ds + |s| 2^-23 + 2^-20 + n 2^-24): the exponent's argument, the
    exponential, and sums of up to n terms, each in the value and in the row sum;
  - lse by ds + |s| 2^-23 + 2^-20 + n 2^-24, the mass by dp times itself;
  - out by 2^-8 |out| (its rounding to bf16) + (2^-8 + dp + n 2^-24) sum P |V|
    (P's rounding to bf16, and the sums);
  - below that, the exponential gives 0 for results under 2^-126.  They are taken
    relative to a reference that is at most the row's maximum, so a row's sum
    is at least 1 and a probability under 2^-126 may count as 0: 2^-126 sum |V|
    of out, and of the mass 2^-126 for every query row.
"""
import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
import workloads as W
from gpu_util import note
from oracle import quant as Q
from oracle import rope as R

pytestmark = pytest.mark.gpu


def cap32(n):
    return max(32, -(-n // 32) * 32)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def u8(t):
    return t.view(torch.uint8).cpu().numpy()


def status_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def rows_like_a_models(rng, shape):
    """Channels of different size, rows of different size."""
    return (rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[-1]))
            * np.exp(0.7 * rng.standard_normal(shape[:-1] + (1,))))


def values(codes, exps):
    """float64 values of a cache's tensors."""
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(exps.double() - 127.0)[..., None]


def to_cache(x):
    """A padded 8-bit side (codes uint8, exponents) of float64 rows, on the device."""
    c, e = Q.encode(x)
    return dev(c), dev(e)


def paged(t, table, n_pages, P, fill):
    """Scatter a padded tensor [B][Hkv][rows][...] into pages; unused bytes are `fill`."""
    B, H, n = t.shape[:3]
    pool = torch.full((n_pages, H, P) + t.shape[3:], fill, dtype=t.dtype, device=t.device)
    for b in range(B):
        for p, pg in enumerate(table[b]):
            if pg >= 0 and p * P < n:
                rows = t[b, :, p * P:(p + 1) * P]
                pool[pg, :, :rows.shape[1]] = rows
    return pool


# ------------------------------------------------------------------- rows --
SPECIAL = [0.0, -0.0, 448.0, 464.0, 1e-40, 3e38, -3e38, np.nan, np.inf, -np.inf, 2.0 ** -133, 17.0, 19.0]


def special_rows(rng, n, D):
    x = rows_like_a_models(rng, (n, D))
    x[0] = 0.0
    x[1] = 1e-39
    x[2] = 3.3e38 * np.sign(x[2])
    x[3, 3] = np.nan
    x[4, 4] = np.inf
    x[5] = np.nan
    x[6] = 2.0 ** rng.integers(-12, 3, D) * 1.0625       # halfway values after scaling
    x[7] = 448.0
    x[8] = -17.0
    for i, s in enumerate(SPECIAL):
        x[9 + i, i] = s
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_quantise_special_rows_bit_exact(dtype, D):
    rng = np.random.default_rng(D)
    n = 77
    x, y = special_rows(rng, n, D), special_rows(rng, n, D)[::-1]
    cast = Q.bf16 if dtype == "bf16" else (lambda a: a.astype(np.float32).astype(np.float64))
    with np.errstate(over="ignore"):
        x, y = cast(x), cast(y)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (dev(a.reshape(1, 1, n, D)).to(tdt) for a in (x, y))
    cap = cap32(n)
    cache = [torch.full(s, 0xAB, dtype=torch.uint8, device="cuda") for s in ((1, 1, cap, D), (1, 1, cap)) * 2]
    note(f"quantise special rows {dtype} D={D}")
    st = status_word()
    pv.quantize_kv(k, v, torch.tensor([n], dtype=torch.int32, device="cuda"), *cache, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for a, c, e in ((x, cache[0], cache[1]), (y, cache[2], cache[3])):
        rc, re = Q.encode(a)
        assert np.array_equal(u8(e)[0, 0, :n], re)
        off = np.argwhere(u8(c)[0, 0, :n] != rc)
        assert not len(off), [(tuple(i), a[tuple(i)], u8(c)[0, 0][tuple(i)], rc[tuple(i)]) for i in off[:4]]
        assert np.all(u8(c)[0, 0, n:] == 0xAB) and np.all(u8(e)[0, 0, n:] == 0xAB)


@pytest.mark.parametrize("L,B,Hkv,D,lens,src_cap,P", [
    (1, 1, 1, 64, [1], 1, 0), (3, 2, 4, 128, [70, 0], 71, 0), (2, 3, 2, 64, [5, 200, 64], 200, 32),
    (28, 1, 4, 128, [301], 333, 64), (1, 4, 8, 128, [33, 1, 512, 31], 600, 256),
])
def test_quantise_stacked(L, B, Hkv, D, lens, src_cap, P):
    rng = np.random.default_rng(L + B + D)
    x = [Q.bf16(rows_like_a_models(rng, (L, B, Hkv, src_cap, D))) for _ in range(2)]
    k, v = (dev(a).to(torch.bfloat16) for a in x)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    note(f"quantise stacked L{L} B{B} H{Hkv} D{D} lens{lens} P{P}")
    st = status_word()
    if P:
        table, n_pages = W.page_table(np.array(lens), P, seed=4)
        shape = (L, n_pages, Hkv, P)
    else:
        shape = (L, B, Hkv, cap32(max(lens)))
    cache = [torch.full(s, 0xC3, dtype=torch.uint8, device="cuda") for s in (shape + (D,), shape) * 2]
    if P:
        pv.quantize_kv_paged(k, v, ln, *cache, dev(table), status=st)
    else:
        pv.quantize_kv(k, v, ln, *cache, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for a, c, e in ((x[0], u8(cache[0]), u8(cache[1])), (x[1], u8(cache[2]), u8(cache[3]))):
        rc, re = Q.encode(a)
        seen = np.zeros(e.shape, bool)
        for b, n in enumerate(lens):
            for i in range(n):
                at = (slice(None), table[b, i // P], slice(None), i % P) if P else (slice(None), b, slice(None), i)
                assert np.array_equal(c[at], rc[:, b, :, i]) and np.array_equal(e[at], re[:, b, :, i])
                seen[at] = True
        assert np.all(c[~seen] == 0xC3) and np.all(e[~seen] == 0xC3)


def test_quantise_flags_lengths_and_pages():
    k = torch.randn((1, 2, 40, 64), device="cuda")
    cache = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((1, 2, 32, 64), (1, 2, 32)) * 2]
    for n, flagged in ((41, True), (33, True), (-1, True), (32, False)):
        st = status_word()
        note(f"quantise length {n} of 40 rows into 32")
        pv.quantize_kv(k, k, torch.tensor([n], dtype=torch.int32, device="cuda"), *cache, status=st)
        assert bool(int(st.item()) & pv.PVLM_DEV_RANGE) == flagged
    pool = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((3, 2, 32, 64), (3, 2, 32)) * 2]
    st = status_word()
    pv.quantize_kv_paged(k, k, torch.tensor([40], dtype=torch.int32, device="cuda"), *pool,
                         torch.tensor([[1, 9]], dtype=torch.int32, device="cuda"), status=st)
    assert int(st.item()) & pv.PVLM_DEV_RANGE
    assert pool[1][1].any() and not pool[1][[0, 2]].any()


APPENDS = [
    # B, T, Hq, Hkv, D, ctx, sections, P
    (1, 1, 1, 1, 64, [0], None, 0),
    (1, 6, 28, 4, 128, [6432], None, 32),
    (3, 9, 40, 8, 128, [8185, 30, 4100], (16, 24, 24), 32),
    (2, 5, 4, 1, 64, [100, 3], (8, 12, 12), 0),
    (2, 300, 8, 2, 128, [0, 17], None, 0),
    (1, 1, 64, 8, 128, [131071], None, 0),
    (2, 33, 7, 1, 64, [31, 96], None, 64),
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: f"B{c[0]}T{c[1]}H{c[2]}/{c[3]}D{c[4]}P{c[7]}")
def test_append_bit_exact(case):
    """q_out and the rows are those of the bf16 append, quantised."""
    B, T, Hq, Hkv, D, ctx, sections, P = case
    rng = np.random.default_rng(sum(ctx) + T)
    q, kn, vn = (dev(rows_like_a_models(rng, (B, T, h, D))).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    vn[0, 0, 0, 3] = float("nan")
    vn[0, T - 1, Hkv - 1] = 0.0
    ctx_np = np.array(ctx, np.int32)
    t0 = ctx_np[:, None] + np.arange(T)[None]
    pos = t0 if sections is None else np.stack([t0, np.maximum(t0 - 5, 0), t0 + 9])
    pos, ctx_t = dev(pos.astype(np.int32)), dev(ctx_np)
    kw = dict(base=1.0e6, sections=sections)
    n_cap = cap32(max(ctx) + T)
    note(f"append q8 {case}")
    st = status_word()
    if P:
        table, n_pages = W.page_table(ctx_np.astype(np.int64) + T, P, seed=5)
        shape = (n_pages, Hkv, P)
        cache = [torch.full(s, 0x5A, dtype=torch.uint8, device="cuda") for s in (shape + (D,), shape) * 2]
        qo = pv.rope_append_q8_paged(q, kn, vn, pos, ctx_t, *cache, dev(table), status=st, **kw)
    else:
        shape = (B, Hkv, n_cap)
        cache = [torch.full(s, 0x5A, dtype=torch.uint8, device="cuda") for s in (shape + (D,), shape) * 2]
        qo = pv.rope_append_q8(q, kn, vn, pos, ctx_t, *cache, status=st, **kw)
    k16 = torch.zeros((B, Hkv, n_cap, D), dtype=torch.bfloat16, device="cuda")
    v16 = torch.zeros_like(k16)
    q16 = pv.rope_append(q, kn, vn, pos, ctx_t, k16, v16, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert torch.equal(qo.view(torch.int16), q16.view(torch.int16))
    # the rotation itself, against the oracle: one rounding to bf16
    rq = R.rotate(q.double().cpu().numpy(), R.pair_positions(pos.cpu().numpy(), D, sections)[:, :, None], 1.0e6)
    assert np.all(np.abs(qo.double().cpu().numpy() - rq) <= 2.0 ** -8 * np.abs(rq) + 1e-30)
    for src, c, e in ((k16, u8(cache[0]), u8(cache[1])), (v16, u8(cache[2]), u8(cache[3]))):
        seen = np.zeros(e.shape, bool)
        for b in range(B):
            i = np.arange(ctx[b], ctx[b] + T)
            rc, re = Q.encode(src[b, :, ctx[b]:ctx[b] + T].double().cpu().numpy())
            at = (table[b, i // P], slice(None), i % P) if P else (b, slice(None), i)
            got_c, got_e = c[at].swapaxes(0, 1), e[at].swapaxes(0, 1)   # (the indexed axes come first)
            assert np.array_equal(got_c, rc) and np.array_equal(got_e, re)
            seen[at] = True
        assert np.all(c[~seen] == 0x5A) and np.all(e[~seen] == 0x5A)
    # in place
    again = q.clone()
    args = (again, kn, vn, pos, ctx_t, *cache)
    (pv.rope_append_q8_paged(*args, dev(table), q_out=again, **kw) if P
     else pv.rope_append_q8(*args, q_out=again, **kw))
    torch.cuda.synchronize()
    assert torch.equal(again.view(torch.int16), q16.view(torch.int16))


def test_append_flags_context_and_pages():
    q = torch.randn((1, 4, 2, 64), device="cuda").to(torch.bfloat16)
    kn = torch.randn((1, 4, 1, 64), device="cuda").to(torch.bfloat16)
    pos = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    for ctx, first in ((29, 28), (-3, 0)):
        cache = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((1, 1, 32, 64), (1, 1, 32)) * 2]
        st = status_word()
        note(f"append context {ctx} of 32 rows")
        pv.rope_append_q8(q, kn, kn, pos, torch.tensor([ctx], dtype=torch.int32, device="cuda"), *cache,
                          base=1e4, status=st)
        assert int(st.item()) & pv.PVLM_DEV_RANGE
        assert cache[1][0, 0, first:first + 4].all() and int((cache[1] != 0).sum()) == 4
    pool = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((3, 1, 32, 64), (3, 1, 32)) * 2]
    st = status_word()
    note("append page entry outside the pool")
    pv.rope_append_q8_paged(q, kn, kn, pos, torch.tensor([30], dtype=torch.int32, device="cuda"), *pool,
                            torch.tensor([[1, 3]], dtype=torch.int32, device="cuda"), base=1e4, status=st)
    assert int(st.item()) & pv.PVLM_DEV_RANGE
    assert int((pool[1] != 0).sum()) == 2 and pool[1][1, 0, 30:].all()


# ----------------------------------------------------------------- verify --
def reference(q, K, V, ctx, scale):
    """float64 attention of q [B][T][Hq][D] (device) over K, V [B][Hkv][n][D], and the bounds above."""
    B, T, Hq, D = q.shape
    Hkv, n_cap = K.shape[1], K.shape[2]
    G = Hq // Hkv
    f = dict(dtype=torch.float64, device=q.device)
    out, lse, mass = torch.zeros((B, T, Hq, D), **f), torch.zeros((B, Hq, T), **f), torch.zeros((B, n_cap), **f)
    b_out, b_lse, b_mass = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(mass)
    qd = q.double()
    for b, c in enumerate(ctx):
        n = c + T
        t = torch.arange(T, device=q.device).repeat_interleave(G)
        hidden = torch.arange(n, device=q.device)[None] > c + t[:, None]
        for g in range(Hkv):
            k, v = K[b, g, :n], V[b, g, :n]
            hs = slice(g * G, (g + 1) * G)
            x = qd[b, :, hs].reshape(T * G, D)
            s = (scale * x @ k.t()).masked_fill(hidden, -torch.inf)
            ds = scale * (D + 4) * 2.0 ** -24 * x.abs() @ k.abs().t()
            ds = (ds + s.abs() * 2.0 ** -23).masked_fill(hidden, 0.0)
            ds = ds.amax(dim=-1, keepdim=True) + 2.0 ** -20 + n * 2.0 ** -24
            z = torch.logsumexp(s, dim=-1, keepdim=True)
            p = torch.exp(s - z)
            dp = 2 * ds
            o = p @ v
            out[b, :, hs] = o.view(T, G, D)
            b_out[b, :, hs] = (2.0 ** -8 * o.abs() + (2.0 ** -8 + dp + n * 2.0 ** -24)
                               * (p @ v.abs()) + 2.0 ** -126 * v.abs().sum(dim=0)).view(T, G, D)
            lse[b, hs] = z.view(T, G).t()
            b_lse[b, hs] = ds.view(T, G).t()
            mass[b, :n] += p.sum(dim=0)
            b_mass[b, :n] += (dp * p).sum(dim=0)
    return (out, lse, mass), (b_out, b_lse, b_mass + 2.0 ** -126 * Hq * T)


def check(got, want, bound, name):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    bad &= ~(torch.isnan(got) & torch.isnan(want))
    at = [tuple(i) for i in torch.nonzero(bad)[:4].tolist()]
    assert not at, (f"{name}: {int(bad.sum())} of {bad.numel()} beyond the bound, e.g. "
                    + str([(i, float(got[i]), float(want[i]), float(bound[i])) for i in at]))


def queries(rng, B, T, Hq, D, scale_up=1.0):
    return dev(rows_like_a_models(rng, (B, T, Hq, D)) * scale_up).to(torch.bfloat16)


def run_verify(q, cache, ctx, scale=None, P=0, seed=0, max_ctx=None, want_mass=True, garbage=True):
    """The call on a padded and (P) paged cache whose unwritten rows hold NaN codes and exponent 255."""
    B, T, Hq, D = q.shape
    cache = [c.clone() for c in cache]
    if garbage:
        for b, c in enumerate(ctx):
            for t, x in zip(cache, (0x7f, 0xff) * 2):
                t[b, :, c + T:] = x
    st = status_word()
    ctx_t = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    kw = dict(scale=scale, status=st, want_mass=want_mass)
    got = pv.verify_attn_q8(q, *cache, ctx_t, max_ctx=max_ctx, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    if P:
        table, n_pages = W.page_table(np.array(ctx) + T, P, seed=seed)
        pools = [paged(t, table, n_pages, P, x) for t, x in zip(cache, (0x7f, 0xff) * 2)]
        # an equal max_ctx gives the padded call's plan, so the results are the same bits
        mc = max(ctx) if max_ctx is None else max_ctx
        got = pv.verify_attn_q8(q, *cache, ctx_t, max_ctx=mc, **kw)
        pg = pv.verify_attn_q8_paged(q, *pools, dev(table), ctx_t, max_ctx=mc, **kw)
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


def random_cache(rng, B, Hkv, rows, D, spread=0.0):
    side = []
    for _ in range(2):
        x = rows_like_a_models(rng, (B, Hkv, cap32(rows), D))
        if spread:
            x *= 2.0 ** rng.uniform(-spread, spread, x.shape[:-1] + (1,))
        side += to_cache(x)
    return side


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
    (4, 9, 28, 4, 128, [100, 900, 3, 1500], 32),    # empty chunks
    (1, 17, 64, 8, 128, [5000], 32),                # 9 row tiles in one workgroup
    (16, 1, 28, 4, 128, [97 * i for i in range(16)], 64),   # a decode batch, one sequence empty but for its token
    (1, 1, 8, 8, 64, [63], 0), (1, 1, 8, 8, 64, [62], 0), (1, 1, 8, 8, 64, [64], 0),
    (1, 5, 4, 1, 64, [255], 0), (1, 5, 4, 1, 64, [252], 0), (1, 6, 4, 4, 128, [122], 0),
    (1, 11, 6, 1, 128, [777], 0), (1, 15, 6, 1, 64, [1000], 32),      # 5 and 6 tiles
    (1, 16, 7, 1, 128, [500], 0), (1, 16, 8, 1, 64, [600], 0),        # 7 and 8 tiles
    (1, 9, 5, 1, 128, [400], 0), (1, 9, 7, 1, 64, [400], 32),         # 3 and 4 tiles
]


@pytest.mark.parametrize("case", VERIFIES, ids=lambda c: f"B{c[0]}T{c[1]}H{c[2]}/{c[3]}D{c[4]}c{c[5][0]}P{c[6]}")
def test_verify_shapes(case):
    B, T, Hq, Hkv, D, ctx, P = case
    rng = np.random.default_rng(sum(ctx) + 7 * T + D)
    q, cache = queries(rng, B, T, Hq, D), random_cache(rng, B, Hkv, max(ctx) + T, D)
    note(f"verify q8 {case}")
    out, mass, lse = run_verify(q, cache, ctx, P=P, seed=B)
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, D ** -0.5)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")
    check(mass[:, :rm.shape[1]], rm, bm, "mass")
    for b, c in enumerate(ctx):
        assert not mass[b, c + T:].any()


def test_verify_long_contexts():
    """131K rows, 136 query rows a KV head; and a decode step over the same cache."""
    rng = np.random.default_rng(3)
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    B, T, Hq, Hkv, D, ctx = 1, 17, 16, 2, 128, 131072 - 17
    x = [torch.randn((B, Hkv, 131072, D), device="cuda", generator=g) for _ in range(2)]
    cache = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((B, Hkv, 131072, D), (B, Hkv, 131072)) * 2]
    pv.quantize_kv(*x, torch.tensor([131072], dtype=torch.int32, device="cuda"), *cache)
    q = queries(rng, B, T, Hq, D)
    K, V = values(*cache[:2]), values(*cache[2:])
    note("verify q8 131K, T = 17")
    out, mass, lse = run_verify(q, cache, [ctx])
    (ro, rl, rm), (bo, bl, bm) = reference(q, K, V, [ctx], D ** -0.5)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")
    check(mass, rm, bm, "mass")
    one = q[:, :1].contiguous()
    note("verify q8 131K, T = 1")
    out, _, lse = run_verify(one, cache, [131071], want_mass=False)
    (ro, rl, _), (bo, bl, _) = reference(one, K, V, [131071], D ** -0.5)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")


def test_verify_offsets_past_32_bits():
    """A pool of more than 2^32 bytes of codes: the sequence's pages are its last ones."""
    P, Hkv, D, n_pages = 1024, 8, 128, 4200      # 4.4 GB of codes a side
    rng = np.random.default_rng(5)
    ctx, T, Hq = [4000], 3, 16
    side = random_cache(rng, 1, Hkv, ctx[0] + T, D)
    pools = [torch.zeros((n_pages, Hkv, P) + t.shape[3:], dtype=torch.uint8, device="cuda") for t in side]
    table = torch.tensor([[n_pages - 1 - 2 * i for i in range(4)]], dtype=torch.int32, device="cuda")
    for i in range(4):
        for t, p in zip(side, pools):
            rows = t[0, :, i * P:(i + 1) * P]
            p[int(table[0, i]), :, :rows.shape[1]] = rows
    q = queries(rng, 1, T, Hq, D)
    ctx_t = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    note("verify q8 over a pool past 4 GB")
    want = pv.verify_attn_q8(q, *side, ctx_t, max_ctx=ctx[0])
    got = pv.verify_attn_q8_paged(q, *pools, table, ctx_t, max_ctx=ctx[0])
    torch.cuda.synchronize()
    assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[2], want[2])
    kn = queries(rng, 1, T, Hkv, D)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[None] + ctx[0]
    pv.rope_append_q8_paged(q, kn, kn, pos, ctx_t, *pools, table, base=1e6)
    pv.rope_append_q8(q, kn, kn, pos, ctx_t, *side, base=1e6)
    page = int(table[0, 3])
    assert torch.equal(pools[0][page, :, 4000 - 3 * P:4003 - 3 * P], side[0][0, :, 4000:4003])
    assert torch.equal(pools[3][page, :, 4000 - 3 * P:4003 - 3 * P], side[3][0, :, 4000:4003])


@pytest.mark.parametrize("D", [64, 128])
def test_verify_wide_ranges(D):
    """Rows whose units differ by 2^24, a key that dwarfs the others (a sink), queries with one large channel."""
    rng = np.random.default_rng(D + 1)
    B, T, Hq, Hkv, ctx = 1, 6, 8, 2, [1500]
    cache = random_cache(rng, B, Hkv, ctx[0] + T, D, spread=12.0)
    ks = random_cache(rng, B, Hkv, ctx[0] + T, D)[:2]
    q = queries(rng, B, T, Hq, D)
    q[..., 5] *= 64.0
    K = values(*ks)
    sink = q[0].double().mean(dim=(0, 1))
    x = K[0].cpu().numpy()
    x[:, 0] = (sink / sink.norm() * 20).cpu().numpy()
    c, e = to_cache(x)
    ks[0][0], ks[1][0] = c, e
    cache = [*ks, *cache[2:]]
    note(f"verify q8 wide ranges D={D}")
    out, mass, lse = run_verify(q, cache, ctx, P=32)
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, D ** -0.5)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")
    check(mass[:, :rm.shape[1]], rm, bm, "mass")


def test_verify_zero_and_extreme_queries():
    rng = np.random.default_rng(12)
    ctx, T, D = [200], 4, 128
    cache = random_cache(rng, 1, 1, ctx[0] + T, D)
    q = queries(rng, 1, T, 4, D)
    q[0, 0] = 0.0                       # the mean of the values
    q[0, 1] *= 2.0 ** -40
    q[0, 2, 0] *= 2.0 ** 20             # one key takes all
    q[0, 3, 0, 1:] *= 2.0 ** -20        # one channel holds all but 2^-20
    note("verify q8 zero, tiny and huge queries")
    out, mass, lse = run_verify(q, cache, ctx)
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, D ** -0.5)
    keep = torch.ones((1, T, 4), dtype=torch.bool, device="cuda")
    keep[0, 2, 0] = False               # (a bound of scores this large says nothing)
    check(out[keep], ro[keep], bo[keep], "out")
    check(lse.transpose(1, 2)[keep], rl.transpose(1, 2)[keep], bl.transpose(1, 2)[keep], "lse")
    top = (q[0, 2, 0].double() @ values(*cache[:2])[0, 0, :ctx[0] + 3].t()).argmax()
    assert torch.allclose(out[0, 2, 0].double(), values(*cache[2:])[0, 0, top], rtol=2.0 ** -7, atol=1e-6)


def test_verify_nan_reaches_only_the_rows_that_see_it():
    rng = np.random.default_rng(6)
    ctx, T, Hq, Hkv, D = [190], 6, 8, 2, 128
    cache = random_cache(rng, 1, Hkv, ctx[0] + T, D)
    q = queries(rng, 1, T, Hq, D)
    clean, _, clse = run_verify(q, cache, ctx, P=32)
    bad = [t.clone() for t in cache]
    bad[2][0, 1, ctx[0] + 3, 17] = 0xff      # V: column 17 of the second KV head, seen by t >= 3
    bad[0][0, 0, ctx[0] + 5, 2] = 0x7f       # K: the first KV head, seen by t = 5
    note("verify q8 NaN in the draft's rows")
    out, mass, lse = run_verify(q, bad, ctx, P=32)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[0, 3:, 4:, 17] = True
    want[0, 5, :4] = True
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(torch.isnan(lse[0]), want[0, :, :, 0].t())
    assert torch.equal(out[~want].view(torch.int16), clean[~want].view(torch.int16))
    bad = [t.clone() for t in cache]
    bad[2][0, 0, 5, 3] = 0x7f                # V in the context: every row of the head
    q2 = q.clone()
    q2[0, 2, 6, 9] = float("inf")            # a query: its own row
    out, mass, lse = run_verify(q2, bad, ctx)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[0, :, :4, 3] = True
    want[0, 2, 6] = True
    assert torch.equal(torch.isnan(out), want)


def test_verify_context_out_of_range_is_clamped_and_flagged():
    rng = np.random.default_rng(9)
    T, Hq, Hkv, D = 3, 4, 2, 64
    cache = random_cache(rng, 2, Hkv, 128, D)
    q = queries(rng, 2, T, Hq, D)
    st = status_word()
    note("verify q8 contexts outside [0, max_ctx]")
    got = pv.verify_attn_q8(q, *cache, torch.tensor([-4, 5000], dtype=torch.int32, device="cuda"), max_ctx=100,
                            status=st)
    want = pv.verify_attn_q8(q, *cache, torch.tensor([0, 100], dtype=torch.int32, device="cuda"), max_ctx=100)
    torch.cuda.synchronize()
    assert int(st.item()) & pv.PVLM_DEV_RANGE
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_verify_bad_page_entry_is_flagged_and_stays_in_the_pool():
    rng = np.random.default_rng(10)
    ctx, T, D = [300, 200], 3, 128
    cache = random_cache(rng, 2, 2, 303, D)
    table, n_pages = W.page_table(np.array(ctx) + T, 32, seed=3)
    pools = [paged(t, table, n_pages, 32, 0x38) for t in cache]
    q = queries(rng, 2, T, 8, D)
    table[1, 2] = n_pages + 7
    st = status_word()
    note("verify q8 page entry outside the pool")
    pv.verify_attn_q8_paged(q, *pools, dev(table), torch.tensor(ctx, dtype=torch.int32, device="cuda"), status=st)
    torch.cuda.synchronize()
    assert int(st.item()) & pv.PVLM_DEV_RANGE


def test_verify_page_table_longer_than_the_staged_entries():
    """256 (sequence, head) groups fill the device: one chunk spans 533 pages."""
    B, T, Hq, D, ctx, P = 1, 1, 256, 64, 17024, 32
    g = torch.Generator(device="cuda")
    g.manual_seed(77)
    q = torch.randn((B, T, Hq, D), device="cuda", generator=g).to(torch.bfloat16)
    x = [torch.randn((B, Hq, ctx + T, D), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]
    n = cap32(ctx + T)
    cache = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((B, Hq, n, D), (B, Hq, n)) * 2]
    pv.quantize_kv(*x, torch.tensor([ctx + T], dtype=torch.int32, device="cuda"), *cache)
    note("verify q8 one chunk of 533 pages")
    run_verify(q, cache, [ctx], P=P, seed=13, garbage=False)


def test_verify_is_the_same_each_time_on_any_stream_and_budget():
    rng = np.random.default_rng(14)
    ctx, T, Hq, Hkv, D = [3000], 9, 64, 8, 128
    cache = random_cache(rng, 1, Hkv, ctx[0] + T, D)
    q = queries(rng, 1, T, Hq, D)
    ctx_t = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    first = pv.verify_attn_q8(q, *cache, ctx_t)
    for _ in range(3):
        for a, b in zip(first, pv.verify_attn_q8(q, *cache, ctx_t)):
            assert torch.equal(a, b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    note("verify q8 on two streams at once")
    outs = []
    for _ in range(4):
        for s in (s1, s2):
            with torch.cuda.stream(s):
                outs.append(pv.verify_attn_q8(q, *cache, ctx_t))
    torch.cuda.synchronize()
    for o in outs:
        for a, b in zip(first, o):
            assert torch.equal(a, b)
    note("verify q8 on a stream of 32 compute units")
    pv.set_stream_cu_budget(s1, 32)
    try:
        with torch.cuda.stream(s1):
            out, mass, lse = pv.verify_attn_q8(q, *cache, ctx_t)
        torch.cuda.synchronize()
    finally:
        pv.set_stream_cu_budget(s1, 0)
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, D ** -0.5)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")
    check(mass, rm, bm, "mass")


def test_workspace_is_checked_and_shared_with_other_calls():
    """A workspace one byte short is refused; one buffer serves the 8-bit call between captured bf16 ones."""
    rng = np.random.default_rng(15)
    ctx, T, Hq, Hkv, D = [900], 5, 8, 2, 128
    cache = random_cache(rng, 1, Hkv, ctx[0] + T, D)
    n_cap = cache[0].shape[2]
    q = queries(rng, 1, T, Hq, D)
    ctx_t = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    need = pv.verify_attn_q8_workspace_size(1, T, Hq, Hkv, D, n_cap, n_cap - T)

    class Short:
        def get(self, n):
            return torch.zeros(n - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(pv.PvlmError) as err:
        pv.verify_attn_q8(q, *cache, ctx_t, ws=Short())
    assert err.value.status == 4
    k16, v16 = values(*cache[:2]).to(torch.bfloat16), values(*cache[2:]).to(torch.bfloat16)
    ws = pv.Workspace()
    ws.get(max(need, pv.verify_attn_workspace_size(pv.PVLM_BF16, 1, T, Hq, Hkv, D, n_cap, n_cap - T)))
    pv.default_status()
    want = pv.verify_attn(q, k16, v16, ctx_t)
    q8 = pv.verify_attn_q8(q, *cache, ctx_t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = pv.verify_attn(q, k16, v16, ctx_t, ws=ws)
    note("one workspace for captured bf16 verify and eager 8-bit verify")
    for _ in range(3):
        g.replay()
        mine = pv.verify_attn_q8(q, *cache, ctx_t, ws=ws)
        torch.cuda.synchronize()
        assert pv.synchronize() == 0
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(mine, q8))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(3, 4), (4, 7), (9, 5), (9, 7), (10, 8), (12, 8), (16, 7), (32, 4), (17, 8), (32, 5),
                                 (32, 6)])
def test_verify_every_number_of_row_tiles(T, G, D):
    """1 to 10 tiles of 16 rows in a workgroup, and 12 over two; pages of one unit."""
    rng = np.random.default_rng(T * G + D)
    ctx = [261, 1337]
    q, cache = queries(rng, 2, T, 2 * G, D), random_cache(rng, 2, 2, max(ctx) + T, D)
    note(f"verify q8 tiles T={T} G={G} D={D}")
    out, mass, lse = run_verify(q, cache, ctx, P=32, seed=T)
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, D ** -0.5)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")
    check(mass[:, :rm.shape[1]], rm, bm, "mass")


@pytest.mark.parametrize("B", [64, 65, 200])
def test_verify_many_sequences(B):
    """More sequences than a wave has lanes; lengths from 0 on, some workgroups with pieces of several sequences."""
    rng = np.random.default_rng(B)
    T, Hq, Hkv, D = 2, 6, 2, 64
    ctx = [int(x) for x in rng.integers(0, 400, B)]
    ctx[0], ctx[B // 2], ctx[B - 1] = 0, 30, 1
    q, cache = queries(rng, B, T, Hq, D), random_cache(rng, B, Hkv, max(ctx) + T, D)
    note(f"verify q8 {B} sequences")
    out, mass, lse = run_verify(q, cache, ctx, P=32, seed=B)
    (ro, rl, rm), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), ctx, D ** -0.5)
    check(out, ro, bo, "out")
    check(lse, rl, bl, "lse")
    check(mass[:, :rm.shape[1]], rm, bm, "mass")


def test_verify_small_probabilities_beside_a_large_one():
    """One key of score 18 (17.5 as its row holds it), 40000 of score 0: each small term is a quarter of the last place of
    the large one, and their sum is 6e-4.  Scores are exact (one channel), so the log-sum-exp is off by five roundings of
    its size (the scale's factor log2(e), two products, two sums) and the logarithm's 2^-20: 6.2e-6.  Rounded away, the
    small terms that share a lane with the large one (600, of 5000 tokens a workgroup) are 9e-6."""
    B, Hkv, D, n = 4, 8, 64, 40000
    x = np.zeros((B, Hkv, cap32(n + 1), D))
    x[:, :, 37, 0] = 17.5
    cache = [*to_cache(x), *to_cache(np.ones_like(x))]
    q = torch.zeros((B, 1, Hkv, D), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    note("verify q8 one large probability among small ones")
    out, mass, lse = run_verify(q, cache, [n] * B, scale=1.0, garbage=False)
    want = np.logaddexp(values(*cache[:2])[0, 0, 37, 0].item(), np.log(n))
    assert (lse.double() - want).abs().max().item() <= 5 * 17.5 * 2.0 ** -24 + 2.0 ** -20
    assert torch.equal(out, torch.ones_like(out))
    p = np.exp(-want)
    assert (mass[:, 1000:n].double() / (Hkv * p) - 1).abs().max().item() <= 2.0 ** -16


def test_verify_calls_of_several_streams_in_one_graph():
    """Two calls with workspaces of their own on two branches of a captured graph, replayed among eager calls."""
    rng = np.random.default_rng(21)
    shapes = [([700, 90], 5, 8, 2, 128), ([3000], 17, 16, 2, 64)]
    work = []
    for ctx, T, Hq, Hkv, D in shapes:
        cache = random_cache(rng, len(ctx), Hkv, max(ctx) + T, D)
        work.append((queries(rng, len(ctx), T, Hq, D), cache, torch.tensor(ctx, dtype=torch.int32, device="cuda"),
                     pv.Workspace()))
    want = [pv.verify_attn_q8(q, *c, n, ws=ws) for q, c, n, ws in work]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    note("verify q8 on two branches of a graph")
    with torch.cuda.graph(g):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        q, c, n, ws = work[0]
        got = [pv.verify_attn_q8(q, *c, n, ws=ws)]
        with torch.cuda.stream(side):
            q, c, n, ws = work[1]
            got.append(pv.verify_attn_q8(q, *c, n, ws=ws))
        main.wait_stream(side)
    for _ in range(3):
        for o in got:
            for t in o:
                t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for o, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))
        for (q, c, n, ws), w in zip(work, want):
            assert all(torch.equal(a, b) for a, b in zip(pv.verify_attn_q8(q, *c, n, ws=ws), w))
        torch.cuda.synchronize()


# ----------------------------------------------------------------- gather --
@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("P,D", [(0, 128), (64, 64), (32, 128)])
def test_gather(dtype, P, D):
    L, B, Hkv = 3, 3, 4
    rng = np.random.default_rng(11 + D)
    rows = np.array([1500, 64, 700])
    n_cap = cap32(int(rows.max()))
    codes = [rng.integers(0, 256, (L, B, Hkv, n_cap, D)).astype(np.uint8) for _ in range(2)]
    exps = [rng.integers(1, 255, (L, B, Hkv, n_cap)).astype(np.uint8) for _ in range(2)]
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
        sides = [np.stack([W.to_pages(a[l], table, n_pages, P) if a.ndim == 5 else
                           W.to_pages(a[l][..., None], table, n_pages, P)[..., 0] for l in range(L)]) for a in sides]
    cache = [dev(a) for a in sides]
    sel = [dev(a) for a in (idx, K, tb, tl)]
    note(f"gather q8 {dtype} P={P} D={D}")
    st = status_word()

    def call(dst=None):
        if P:
            return pv.gather_kv_q8_paged(*cache, dev(table), *sel, dst_cap, dtype=dtype, dst=dst, status=st)
        return pv.gather_kv_q8(*cache, *sel, dst_cap, dtype=dtype, dst=dst, status=st)
    got = call()
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    shape = (L, B, Hkv, dst_cap)
    if dtype is torch.float8_e4m3fn:
        old = [torch.full(s, 0x77, dtype=torch.uint8, device="cuda") for s in (shape + (D,), shape) * 2]
    else:
        old = [torch.full(shape + (D,), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    kept = call(old)
    torch.cuda.synchronize()
    for side in range(2):
        want_c, want_e = np.zeros(shape + (D,), np.uint8), np.zeros(shape, np.uint8)
        live = np.zeros(shape, bool)
        for b in range(B):
            src = np.concatenate([idx[b, :K[b]], tb[b] + np.arange(tl[b])])
            want_c[:, b, :, :len(src)] = codes[side][:, b][:, :, src]
            want_e[:, b, :, :len(src)] = exps[side][:, b][:, :, src]
            live[:, b, :, :len(src)] = True
        live = dev(live)
        if dtype is torch.float8_e4m3fn:
            assert np.array_equal(u8(got[2 * side]), want_c) and np.array_equal(u8(got[2 * side + 1]), want_e)
            assert np.array_equal(u8(kept[2 * side][live]), want_c[live.cpu().numpy()])
            assert bool((kept[2 * side][~live] == 0x77).all()) and bool((kept[2 * side + 1][~live] == 0x77).all())
        else:
            v = dev(Q.decode(want_c, np.where(want_e == 0, 1, want_e)))
            v = torch.where(live[..., None], v, 0.0).to(torch.float32).to(dtype)
            assert torch.equal(torch.isnan(got[side]), torch.isnan(v))
            assert torch.equal(got[side].nan_to_num(nan=1.5), v.nan_to_num(nan=1.5))
            assert torch.equal(kept[side][live].nan_to_num(), got[side][live].nan_to_num())
            assert bool((kept[side][~live] == 7.0).all())


def test_gather_flags_what_is_out_of_range():
    cache = [torch.randint(1, 100, s, dtype=torch.uint8, device="cuda") for s in ((1, 2, 64, 64), (1, 2, 64)) * 2]

    def call(idx, k, tb, tl, cap=32):
        st = status_word()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        r = pv.gather_kv_q8(*cache, i32([idx]), i32([k]), i32([tb]), i32([tl]), cap, status=st)
        return bool(int(st.item()) & pv.PVLM_DEV_RANGE), r
    note("gather q8 indices, counts and tails out of range")
    assert not call([1, 2], 2, 60, 4)[0]
    bad, r = call([1, 64], 2, 60, 4)
    assert bad and not r[1][0, :, 1].any() and r[1][0, :, [0, 2, 3, 4, 5]].all()
    for args in (([1, -1], 2, 60, 4), ([1, 2], 3, 60, 4), ([1, 2], -1, 60, 4), ([1, 2], 2, 65, 0),
                 ([1, 2], 2, 60, 5), ([1, 2], 2, 30, 31), ([1, 2], 2, 30, -1)):
        assert call(*args)[0], args
    pool = [torch.randint(1, 100, s, dtype=torch.uint8, device="cuda") for s in ((2, 2, 32, 64), (2, 2, 32)) * 2]
    st = status_word()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    r = pv.gather_kv_q8_paged(*pool, i32([[1, 2]]), i32([[3, 40]]), i32([2]), i32([5]), i32([1]), 32, status=st)
    assert int(st.item()) & pv.PVLM_DEV_RANGE
    assert torch.equal(r[1][0, :, [0, 2]], pool[1][1, :, [3, 5]]) and not r[1][0, :, 1].any()


# --------------------------------------------------------------- together --
def test_a_decode_loop_as_a_draft_runs_it():
    """Prefill rows quantised, verify with mass, the mass's top rows gathered into an 8-bit compact cache, and decode
    steps over it (append + T = 1), captured in a graph and replayed; every replay equals the eager calls, and
    float64 attention over the values that the cache holds."""
    rng = np.random.default_rng(21)
    B, T, Hq, Hkv, D, m, n = 1, 6, 28, 4, 128, 900, 60
    x = [dev(rows_like_a_models(rng, (B, Hkv, m + n, D))).to(torch.bfloat16) for _ in range(2)]
    cap = cap32(m + n + T)
    cache = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((B, Hkv, cap, D), (B, Hkv, cap)) * 2]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    pv.quantize_kv(*x, i32([m + n]), *cache)
    q, kn, vn = (queries(rng, B, T, h, D) for h in (Hq, Hkv, Hkv))
    ctx = i32([m + n])
    pos = ctx[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
    note("8-bit loop: append, verify, top-k, gather")
    qr = pv.rope_append_q8(q, kn, vn, pos, ctx, *cache, base=1e6)
    out, mass, lse = pv.verify_attn_q8(qr, *cache, ctx)
    (ro, rl, rm), (bo, bl, bm) = reference(qr, values(*cache[:2]), values(*cache[2:]), [m + n], D ** -0.5)
    check(out, ro, bo, "out")
    check(mass, rm, bm, "mass")
    keep = 100
    idx = pv.topk_select(mass[:, :m].contiguous(), i32([m]), i32([keep]), keep)
    assert torch.equal(idx[0].long().cpu(), mass[0, :m].topk(keep).indices.sort().values.cpu())
    draft = pv.gather_kv_q8(*cache, idx, i32([keep]), i32([m]), i32([n]), 192)
    src = torch.cat([idx[0].long(), torch.arange(m, m + n, device="cuda")])
    for a, b in zip(draft, cache):
        assert torch.equal(a.view(torch.uint8)[:, :, :keep + n], b[:, :, src])
    pv.default_status()
    dctx, dpos = i32([keep + n]), i32([[m + n]])
    q1, k1, v1 = (queries(rng, B, 1, h, D) for h in (Hq, Hkv, Hkv))
    qo, do, dl = torch.empty_like(q1), torch.empty_like(q1), torch.empty((B, Hq, 1), device="cuda")
    ws = pv.Workspace()
    ws.get(pv.verify_attn_q8_workspace_size(B, 1, Hq, Hkv, D, 192, 191))

    def step():
        pv.rope_append_q8(q1, k1, v1, dpos, dctx, *draft, base=1e6, q_out=qo)
        pv.verify_attn_q8(qo, *draft, dctx, out=do, lse=dl, want_mass=False, ws=ws)
        dctx.add_(1)
        dpos.add_(1)
    eager = []
    first = [t.view(torch.uint8).clone() for t in draft]
    for _ in range(4):
        step()
        eager.append((do.clone(), dl.clone()))
    torch.cuda.synchronize()
    c = keep + n + 3
    (ro, rl, _), (bo, bl, _) = reference(qo, values(*draft[:2]), values(*draft[2:]), [c], D ** -0.5)
    check(do, ro, bo, "decode out")
    check(dl, rl, bl, "decode lse")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    dctx.fill_(keep + n)
    dpos.fill_(m + n)
    for t, f in zip(draft, first):
        t.view(torch.uint8).copy_(f)
    for i in range(4):
        note(f"8-bit decode step, replay {i}")
        g.replay()
        pv.verify_attn_q8(qr, *cache, ctx)       # the program's own eager work between replays
        torch.cuda.synchronize()
        assert torch.equal(do, eager[i][0]) and torch.equal(dl, eager[i][1])
    assert pv.synchronize() == 0


def test_gather_to_bf16_feeds_the_bf16_calls():
    """Over the values read back, the bf16 verify gives what the 8-bit verify gives over the rows, to rounding."""
    rng = np.random.default_rng(22)
    B, T, Hq, Hkv, D, n = 2, 5, 8, 2, 128, 500
    cache = random_cache(rng, B, Hkv, n, D)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    k, v = pv.gather_kv_q8(*cache, torch.empty((B, 0), dtype=torch.int32, device="cuda"), i32([0, 0]), i32([0, 0]),
                           i32([n, n]), n, dtype=torch.bfloat16)
    assert torch.equal(k.double(), values(*cache[:2])[:, :, :n])
    q = queries(rng, B, T, Hq, D)
    ctx = i32([n - T, 100])
    o16, m16, l16 = pv.verify_attn(q, k, v, ctx)
    o8, m8, l8 = pv.verify_attn_q8(q, *cache, ctx)
    (_, _, _), (bo, bl, bm) = reference(q, values(*cache[:2]), values(*cache[2:]), [n - T, 100], D ** -0.5)
    check(o8, o16.double(), 2 * bo, "out")
    check(l8, l16.double(), 2 * bl, "lse")
    check(m8[:, :n], m16.double(), 2 * bm[:, :n], "mass")


# --------------------------------------------------------------- refusals --
def test_bindings_refuse_what_does_not_fit():
    B, T, Hq, Hkv, D, n = 2, 3, 4, 2, 64, 64
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    cache = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in ((B, Hkv, n, D), (B, Hkv, n)) * 2]
    q, kn = bf(B, T, Hq, D), bf(B, T, Hkv, D)

    def refuse(f, *a, err=ValueError, **kw):
        with pytest.raises(err):
            f(*a, **kw)
    short = [cache[0], cache[1][:, :, :32].contiguous(), *cache[2:]]
    strided = [cache[0].transpose(1, 2).contiguous().transpose(1, 2), *cache[1:]]
    wrong = [cache[0].to(torch.int32), *cache[1:]]
    host = [cache[0].cpu(), *cache[1:]]
    for c in (short, strided, wrong, host):
        refuse(pv.verify_attn_q8, q, *c, i32(B))
        refuse(pv.rope_append_q8, q, kn, kn, i32(B, T), i32(B), *c, base=1e4)
        refuse(pv.quantize_kv, bf(B, Hkv, 10, D), bf(B, Hkv, 10, D), i32(B), *c)
        refuse(pv.gather_kv_q8, *c, i32(B, 4), i32(B), i32(B), i32(B), 32)
    refuse(pv.verify_attn_q8, q.float(), *cache, i32(B))
    refuse(pv.verify_attn_q8, q[:1], *cache, i32(1))
    refuse(pv.verify_attn_q8, q, *cache, i32(B + 1))
    refuse(pv.verify_attn_q8, q, *cache, i32(B), out=bf(B, T, Hq, D + 1))
    refuse(pv.verify_attn_q8, q, *cache, i32(B), mass=torch.zeros((B, n + 1), device="cuda"))
    refuse(pv.verify_attn_q8, q, *cache, i32(B), lse=torch.zeros((B, T, Hq), device="cuda"))
    refuse(pv.verify_attn_q8, q, *cache, i32(B), max_ctx=n, err=pv.PvlmError)
    refuse(pv.verify_attn_q8_paged, q, *cache, None, i32(B), err=TypeError)
    refuse(pv.verify_attn_q8_paged, q, *cache, i32(1, 4), i32(B))
    refuse(pv.rope_append_q8, q, kn, kn[:, :2].contiguous(), i32(B, T), i32(B), *cache, base=1e4)
    refuse(pv.rope_append_q8, q, kn, kn, i32(B, T), i32(B), *cache, base=1e4, sections=(8, 12, 12))
    refuse(pv.rope_append_q8, q, kn, kn, i32(3, B, T), i32(B), *cache, base=1e4, sections=(8, 12, 13),
           err=pv.PvlmError)
    refuse(pv.rope_append_q8, q, kn, kn, i32(B, T), i32(B), *cache, base=1e4, q_out=bf(B, T, Hq))
    refuse(pv.quantize_kv, bf(1, B, Hkv, 10, D), bf(1, B, Hkv, 10, D), i32(B), *cache)
    refuse(pv.quantize_kv, bf(B, Hkv, 10, D).half(), bf(B, Hkv, 10, D).half(), i32(B), *cache)
    refuse(pv.gather_kv_q8, *cache, i32(B, 4), i32(B), i32(B), i32(B), 32, dtype=torch.float16)
    refuse(pv.gather_kv_q8, *cache, i32(B, 4), i32(B), i32(B), i32(B), 33, err=pv.PvlmError)
    refuse(pv.gather_kv_q8, *cache, i32(B, 4), i32(B), i32(B), i32(B), 32, dst=cache)
    refuse(pv.gather_kv_q8, *cache, i32(B, 4), i32(B + 1), i32(B), i32(B), 32)
    off = torch.zeros(B * Hkv * n * D + 1, dtype=torch.uint8, device="cuda")[1:].view(B, Hkv, n, D)
    refuse(pv.verify_attn_q8, q, off, *cache[1:], i32(B), err=pv.PvlmError)      # codes not 16-byte aligned
