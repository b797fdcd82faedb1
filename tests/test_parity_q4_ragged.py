"""GPU parity of the 4-bit verify over sequences with their own numbers of new rows.

The rows that a sequence has are compared with float64 attention of that sequence alone
(the bounds of ``test_parity_q8``); rows of padding are 0 and -inf; and neither what the
padding holds, in q and in the cache, nor page entries past a sequence reach anything.
"""
import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
import workloads as W
from gpu_util import note
from test_parity_pages import Pool, fused_rows
from test_parity_q4 import empty_cache, i32, random_cache, values
from test_parity_q8 import cap32, check, dev, paged, queries, reference, status_word

pytestmark = pytest.mark.gpu

NAN = float("nan")


def check_ragged(got, q, cache, ctx, new):
    """`cache`: padded tensors that hold rows 0 .. ctx[b] + new[b] - 1."""
    out, mass, lse = got
    for b, (c, n) in enumerate(zip(ctx, new)):
        assert not out[b, n:].any() and bool((lse[b, :, n:] == -torch.inf).all())
        seen = c + n if n else 0
        if mass is not None:
            assert not mass[b, seen:].any()
        if not n:
            continue
        side = [t[b:b + 1] for t in cache]
        ref, bound = reference(q[b:b + 1, :n], values(*side[:2]), values(*side[2:]), [c], q.shape[-1] ** -0.5)
        check(out[b:b + 1, :n], ref[0], bound[0], "out")
        check(lse[b:b + 1, :, :n], ref[1], bound[1], "lse")
        if mass is not None:
            check(mass[b:b + 1, :seen], ref[2][:, :seen], bound[2][:, :seen], "mass")


def dirty(q, cache, ctx, new, exps):
    """Copies with NaN in the padding rows of q, and full codes of one exponent past what a sequence has."""
    q, cache = q.clone(), [t.clone() for t in cache]
    for b, (c, n) in enumerate(zip(ctx, new)):
        q[b, n:] = NAN
        for t, x in zip(cache, (0x77, exps) * 2):
            t[b, :, c + n if n else 0:] = x
    return q, cache


def equal(a, b):
    return all(x is y is None or torch.equal(x, y) for x, y in zip(a, b))


CASES = [
    # B, T, Hq, Hkv, D, ctx, new, P
    (1, 5, 8, 2, 128, [0], [1], 32),
    (2, 5, 8, 2, 64, [0, 0], [0, 3], 32),                       # a sequence of nothing at all
    (3, 5, 8, 2, 128, [60, 0, 129], [5, 3, 0], 32),             # one of no new rows
    (4, 9, 7, 1, 128, [31, 32, 33, 27], [1, 0, 9, 5], 32),      # ends at, before and behind a unit
    (3, 32, 20, 1, 64, [30, 333, 1], [1, 17, 31], 64),          # 40 row tiles
    (2, 17, 64, 8, 128, [3000, 700], [1, 9], 32),               # 9 row tiles, shares
    (2, 9, 64, 8, 128, [5000, 4999], [0, 9], 256),              # 5 row tiles; every share of the first one empty
    (4, 2, 28, 4, 128, [2100, 100, 1600, 31], [1, 2, 0, 1], 64),
    (1, 32, 6, 6, 64, [9000], [2], 32),
    (1, 3, 8, 8, 128, [40000], [2], 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[0]}T{c[1]}H{c[2]}/{c[3]}D{c[4]}c{c[5][0]}n{c[6][0]}P{c[7]}")
def test_ragged_shapes(case):
    B, T, Hq, Hkv, D, ctx, new, P = case
    rng = np.random.default_rng(sum(ctx) + 7 * T + D)
    q, cache = queries(rng, B, T, Hq, D), random_cache(rng, B, Hkv, max(ctx) + T, D)
    n, c32, first = i32(new), i32(ctx), None
    mc = max(ctx)
    for exps in (0, 254, 255):                  # 0, infinities in bf16, NaN
        qd, cd = (q, cache) if exps == 0 else dirty(q, cache, ctx, new, exps)
        for mass in (True, False):
            st = status_word()
            note(f"verify q4 ragged {case} exponents {exps} mass {mass}")
            got = pv.verify_attn_q4(qd, *cd, c32, n_new=n, max_ctx=mc, want_mass=mass, status=st)
            torch.cuda.synchronize()
            assert int(st.item()) == 0
            if first is None:
                first = got
                check_ragged(got, q, cache, ctx, new)
            assert equal(got, first if mass else (first[0], None, first[2]))
            if P:                               # tables that end with what a sequence has
                table, n_pages = W.page_table(np.array([x + y if y else 0 for x, y in zip(ctx, new)]), P, seed=B,
                                              max_pages=-(-(mc + T) // P))
                pools = [paged(t, table, n_pages, P, x) for t, x in zip(cd, (0x77, exps) * 2)]
                pg = pv.verify_attn_q4_paged(qd, *pools, dev(table), c32, n_new=n, max_ctx=mc, want_mass=mass, status=st)
                torch.cuda.synchronize()
                assert int(st.item()) == 0
                m = min(first[1].shape[1], table.shape[1] * P)
                assert torch.equal(pg[0], first[0]) and torch.equal(pg[2], first[2])
                if mass:
                    assert torch.equal(pg[1][:, :m], first[1][:, :m]) and not pg[1][:, m:].any()


@pytest.mark.parametrize("B", [65, 200])
def test_ragged_many_sequences(B):
    """Shares that end one sequence and begin the next, empty ones among them."""
    rng = np.random.default_rng(B)
    T, Hq, Hkv, D = 4, 6, 2, 64
    ctx, new = [int(x) for x in rng.integers(0, 400, B)], [int(x) for x in rng.integers(0, T + 1, B)]
    new[0], new[B - 1], ctx[B // 2] = 0, 0, 0
    q, cache = queries(rng, B, T, Hq, D), random_cache(rng, B, Hkv, max(ctx) + T, D)
    qd, cd = dirty(q, cache, ctx, new, 255)
    note(f"verify q4 ragged, {B} sequences")
    got = pv.verify_attn_q4(qd, *cd, i32(ctx), n_new=i32(new))
    check_ragged(got, q, cache, ctx, new)
    assert pv.synchronize() == 0


@pytest.mark.parametrize("T,Hq,Hkv,D,ctx", [(5, 8, 2, 128, [300, 31]), (9, 64, 8, 128, [4000, 700]), (1, 28, 4, 64, [9, 0])])
def test_ragged_with_every_row_is_the_plain_call(T, Hq, Hkv, D, ctx):
    rng = np.random.default_rng(T)
    q, cache = queries(rng, 2, T, Hq, D), random_cache(rng, 2, Hkv, max(ctx) + T, D)
    note(f"verify q4 ragged with all {T} rows")
    want = pv.verify_attn_q4(q, *cache, i32(ctx))
    assert equal(want, pv.verify_attn_q4(q, *cache, i32(ctx), n_new=i32([T, T])))
    # a number of rows out of its range is clamped into it and flagged
    part = pv.verify_attn_q4(q, *cache, i32(ctx), n_new=i32([T, 0]))
    st = status_word()
    got = pv.verify_attn_q4(q, *cache, i32(ctx), n_new=i32([T + 1, -3]), status=st)
    torch.cuda.synchronize()
    assert equal(got, part) and int(st.item()) == pv.PVLM_DEV_RANGE
    assert torch.equal(part[0][0], want[0][0]) and torch.equal(part[1][0], want[1][0]) and not part[1][1].any()


@pytest.mark.parametrize("ctx,T,new,D", [([190, 40], 6, [5, 4], 128), ([31, 3000], 8, [4, 7], 64)])
def test_ragged_nan_reaches_only_the_rows_that_see_it(ctx, T, new, D):
    """In the last and second new row's values, and right behind them (of another sequence's padding)."""
    rng = np.random.default_rng(T)
    q, cache = queries(rng, 2, T, 8, D), random_cache(rng, 2, 2, max(ctx) + T, D)
    n = i32(new)
    clean = pv.verify_attn_q4(q, *cache, i32(ctx), n_new=n)
    bad = [t.clone() for t in cache]
    want = torch.zeros((2, T, 8, D), dtype=torch.bool, device="cuda")
    for b in range(2):
        bad[3][b, 1, ctx[b] + 1, 1] = 255
        bad[3][b, 0, ctx[b] + new[b] - 1, 0] = 255
        bad[3][b, 0, ctx[b] + new[b], 1] = 255
        want[b, 1:new[b], 4:, 32:64] = True
        want[b, new[b] - 1, :4, :32] = True
    note("verify q4 ragged, NaN in the new rows")
    got = pv.verify_attn_q4(q, *bad, i32(ctx), n_new=n)
    assert torch.equal(torch.isnan(got[0]), want) and torch.equal(got[0][~want], clean[0][~want])
    assert equal(got[1:], clean[1:])


def test_refuses_a_number_of_rows_that_does_not_fit():
    q, cache = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda"), empty_cache((2, 2, 64), 64)
    n = i32([1, 1])
    for bad in (i32([1]), n.long(), n.cpu(), i32([[1, 1]]), torch.zeros(4, dtype=torch.int32, device="cuda")[::2]):
        with pytest.raises(ValueError):
            pv.verify_attn_q4(q, *cache, n, n_new=bad)
        with pytest.raises(ValueError):
            pv.verify_attn_q4_paged(q, *cache, i32([[0, 1], [1, 0]]), n, n_new=bad)
    with pytest.raises(TypeError):
        pv.verify_attn_q4(q, *cache, n, n_new=[1, 1])


def test_a_ragged_serving_step_as_a_graph():
    """Tables grown for the rows that a sequence has, their slots, the append, the verify and the cut, captured in one graph
    and replayed: every replay equals the calls made one by one on a copy, and float64 attention over the rows that
    there are.  The pool begins as NaN, and the append's queries are a new tensor's, whose padding nobody writes."""
    rng = np.random.default_rng(32)
    B, T, Hq, Hkv, D, P, max_pages, n_pages = 4, 5, 8, 2, 128, 32, 9, 40
    rot = pv.Rotary(rot_dim=D, base=1e6)
    ctx0, new0 = [60, 0, 129, 31], [5, 3, 0, 1]
    pool = Pool(B, P, max_pages, n_pages, seed=3)
    pool.resize(ctx0)
    held, table, free, n_free = pool.d
    cache = empty_cache((n_pages, Hkv, P), D, 0xff)
    slots, pos, _, _ = pv.slot_map(i32([0] * B), i32(ctx0), sum(ctx0), page_size=P, n_pages=n_pages, page_table=table)
    pv.rotary_append_q4(*fused_rows(rng, sum(ctx0), Hq, Hkv, D, torch.bfloat16), pos, slots, *cache, rotary=rot)
    ctx, new, accepted = i32(ctx0), i32(new0), i32([2, 3, 0, 1])
    q, k, v = fused_rows(rng, B * T, Hq, Hkv, D, torch.bfloat16)
    want_len, granted, kept = i32([0] * B), i32([9] * B), i32([9] * B)
    pv.default_status()

    def step(held, table, free, n_free, cache, ctx):
        torch.add(ctx, new, out=want_len)
        pv.pages_resize(want_len, held, table, free, n_free, page_size=P, granted=granted)
        slots, pos, _, _ = pv.slot_map(ctx, new, B * T, page_size=P, n_pages=n_pages, page_table=table, rows_per_seq=T)
        turned = torch.empty((B * T, Hq, D), dtype=torch.bfloat16, device="cuda")
        turned.fill_(NAN)                       # (the worst that new memory may hold)
        pv.rotary_append_q4(q, k, v, pos, slots, *cache, rotary=rot, q_out=turned)
        out, mass, lse = pv.verify_attn_q4_paged(turned.view(B, T, Hq, D), *cache, table, ctx, n_new=new)
        seen = table.clone()
        ctx.add_(accepted)
        pv.pages_resize(ctx, held, table, free, n_free, page_size=P, granted=kept)
        return out, mass, lse, seen, turned
    copy = [t.clone() for t in (held, table, free, n_free, *cache, ctx)]
    warm = [t.clone() for t in copy]
    step(*warm[:4], warm[4:8], warm[8])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(held, table, free, n_free, cache, ctx)
    for i in range(4):
        note(f"ragged serving step, replay {i}")
        at = ctx.tolist()
        g.replay()
        torch.cuda.synchronize()
        eager = step(*copy[:4], copy[4:8], copy[8])
        torch.cuda.synchronize()
        for a, b in zip(got[:4], eager[:4]):
            assert torch.equal(a, b)
        for a, b in zip((held, table, free, n_free, *cache, ctx), copy):
            assert torch.equal(a, b)
        n = cap32(max(at) + T)
        pad = [torch.full((B, Hkv, n, t.shape[-1]), 0xff, dtype=torch.uint8, device="cuda") for t in cache]
        for b in range(B):
            for j in range(-(-(at[b] + new0[b]) // P)):
                for x, t in zip(pad, cache):
                    x[b, :, j * P:(j + 1) * P] = t[got[3][b, j].item()][:, :n - j * P]
        check_ragged((got[0], got[1][:, :n], got[2]), got[4].view(B, T, Hq, D), pad, at, new0)
        assert ctx.tolist() == [x + y for x, y in zip(at, accepted.tolist())]
    assert pv.synchronize() == 0
