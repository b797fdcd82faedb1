"""GPU parity of the 8-bit calls in the ways that programs make them: captured
graphs beside each other, prompts, calls without mass or log-sum-exp, 32-bit
sources.  Reference and bounds are those of ``test_parity_q8``."""
import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
import workloads as W
from gpu_util import note
from oracle import quant as Q
from test_parity_q8 import cap32, dev, queries, random_cache, rows_like_a_models, run_verify, status_word, u8
from test_parity_q8 import test_append_bit_exact as append_bit_exact

pytestmark = pytest.mark.gpu


def test_graphs_of_one_capture_stream_replay_together():
    """Two graphs captured one after the other on torch's capture stream, without workspaces of their own, replayed on two
    streams at once and beside eager calls: every result is the eager one's."""
    rng = np.random.default_rng(31)
    shapes = [([9000], 9, 64, 8, 128), ([7000, 30], 6, 28, 4, 128)]
    work = [(queries(rng, len(c), T, Hq, D), random_cache(rng, len(c), Hkv, max(c) + T, D),
             torch.tensor(c, dtype=torch.int32, device="cuda")) for c, T, Hq, Hkv, D in shapes]
    pv.default_status()
    want = [[t.clone() for t in pv.verify_attn_q8(q, *c, n)] for q, c, n in work]
    torch.cuda.synchronize()
    graphs, outs = [], []
    note("verify q8: two graphs of one capture stream")
    for q, c, n in work:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(pv.verify_attn_q8(q, *c, n))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(4):
        note(f"verify q8: two graphs together, round {rep}")
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                for _ in range(5):
                    g.replay()
        eager = [pv.verify_attn_q8(q, *c, n) for q, c, n in work]
        torch.cuda.synchronize()
        for got in (outs, eager):
            for o, w in zip(got, want):
                assert all(torch.equal(a, b) for a, b in zip(o, w))
    assert pv.synchronize() == 0


@pytest.mark.parametrize("B,T,Hq,Hkv,D,ctx,spare", [(2, 9, 20, 4, 128, [800, 31], 3000), (1, 32, 20, 1, 64, [333], 9000),
                                                    (1, 1, 8, 8, 64, [0], 64)])
def test_a_cache_with_much_room_takes_the_workspace_of_its_contexts(B, T, Hq, Hkv, D, ctx, spare):
    """A capacity beyond the longest context changes neither the workspace nor the results, and nothing is written past
    the workspace's end."""
    rng = np.random.default_rng(spare)
    tight = -(-(max(ctx) + T) // 32) * 32
    cache = random_cache(rng, B, Hkv, tight + spare, D)
    q = queries(rng, B, T, Hq, D)
    n = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    n_cap = cache[0].shape[2]
    need = pv.verify_attn_q8_workspace_size(B, T, Hq, Hkv, D, n_cap, max(ctx))
    assert need == pv.verify_attn_q8_workspace_size(B, T, Hq, Hkv, D, tight, max(ctx))
    buf = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")

    class Exact:
        def get(self, nbytes):
            assert nbytes == need
            return buf[:need]
    note(f"verify q8 with {spare} spare rows")
    got = pv.verify_attn_q8(q, *cache, n, max_ctx=max(ctx), ws=Exact())
    want = pv.verify_attn_q8(q, *[c[:, :, :tight].contiguous() for c in cache], n, max_ctx=max(ctx))
    torch.cuda.synchronize()
    assert bool((buf[need:] == 0xA5).all())
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    assert torch.equal(got[1][:, :tight], want[1]) and not got[1][:, tight:].any()


PROMPTS = [
    # B, T, Hq, Hkv, D, ctx, sections, P: more than 1024 passes over heads, so a workgroup takes every head of a row
    (1, 700, 28, 4, 128, [0], None, 0),
    (1, 2049, 64, 8, 128, [0], (16, 24, 24), 32),
    (2, 600, 8, 4, 64, [0, 17], None, 64),
    (1, 1100, 40, 8, 64, [5], (8, 12, 12), 0),
    (3, 341, 20, 4, 128, [0, 0, 90], None, 256),
    (1, 512, 16, 8, 128, [0], None, 0), (1, 513, 16, 8, 128, [0], None, 0),     # 1024 passes, and two more
]


@pytest.mark.parametrize("case", PROMPTS, ids=lambda c: f"B{c[0]}T{c[1]}H{c[2]}/{c[3]}D{c[4]}P{c[7]}")
def test_append_of_a_prompt_bit_exact(case):
    append_bit_exact(case)


@pytest.mark.parametrize("L,B,Hkv,D,lens,src_cap,P", [
    (3, 2, 4, 128, [70, 0], 71, 0), (2, 3, 2, 64, [5, 200, 64], 200, 32), (4, 1, 8, 64, [1], 1, 0),
    (5, 2, 5, 128, [301, 17], 333, 64),
])
def test_quantise_32_bit_rows(L, B, Hkv, D, lens, src_cap, P):
    rng = np.random.default_rng(L + B + D)
    x = [rows_like_a_models(rng, (L, B, Hkv, src_cap, D)).astype(np.float32) for _ in range(2)]
    note(f"quantise fp32 L{L} B{B} H{Hkv} D{D} lens{lens} P{P}")
    st = status_word()
    table, n_pages = W.page_table(np.array(lens), P, seed=6) if P else (None, 0)
    shape = (L, n_pages, Hkv, P) if P else (L, B, Hkv, cap32(max(lens)))
    cache = [torch.full(s, 0xC3, dtype=torch.uint8, device="cuda") for s in (shape + (D,), shape) * 2]
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if P:
        pv.quantize_kv_paged(dev(x[0]), dev(x[1]), ln, *cache, dev(table), status=st)
    else:
        pv.quantize_kv(dev(x[0]), dev(x[1]), ln, *cache, status=st)
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


@pytest.mark.parametrize("T,D,ctx,P", [(5, 64, [300, 7], 0), (9, 128, [1300, 64], 32), (17, 128, [5000, 4999], 64),
                                       (32, 64, [90, 200], 0), (1, 128, [700, 0], 32)])
def test_verify_without_mass_or_lse_gives_the_same_outputs(T, D, ctx, P):
    rng = np.random.default_rng(T)
    q, cache = queries(rng, 2, T, 14, D), random_cache(rng, 2, 2, max(ctx) + T, D)
    n = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    note(f"verify q8 T={T} D={D} without mass, without lse")
    out, mass, lse = run_verify(q, cache, ctx, P=P, seed=T)
    bare, none, lse2 = run_verify(q, cache, ctx, P=P, seed=T, want_mass=False)
    assert none is None and torch.equal(bare, out) and torch.equal(lse2, lse)
    mc = max(ctx) if P else None
    for want_mass in (False, True):
        o, m, l = pv.verify_attn_q8(q, *cache, n, max_ctx=mc, want_mass=want_mass, want_lse=False)
        assert l is None and torch.equal(o, out)
        assert m is None or torch.equal(m, mass)
    given = [torch.full_like(t, 7.0) for t in (out, mass, lse)]
    got = pv.verify_attn_q8(q, *cache, n, max_ctx=mc, out=given[0], mass=given[1], lse=given[2])
    for a, b, w in zip(got, given, (out, mass, lse)):
        assert a is b and torch.equal(a, w)


@pytest.mark.parametrize("B,T,Hq,Hkv,D,ctx,P", [(1, 8, 4, 1, 64, [63], 32), (2, 32, 20, 1, 64, [90, 33], 0),
                                                (2, 9, 64, 8, 128, [2000, 31], 64), (1, 17, 32, 2, 128, [4095], 0)])
def test_nan_in_every_draft_row_reaches_the_rows_that_see_it(B, T, Hq, Hkv, D, ctx, P):
    """One KV head's values: row ctx + j has a NaN in column j (mod D); a query row t has the columns 0 .. t of it."""
    rng = np.random.default_rng(T + D)
    cache = random_cache(rng, B, Hkv, max(ctx) + T, D)
    q = queries(rng, B, T, Hq, D)
    clean = run_verify(q, cache, ctx, P=P, seed=3)
    g, G = Hkv - 1, Hq // Hkv
    want = torch.zeros((B, T, Hq, D), dtype=torch.bool, device="cuda")
    for b, c in enumerate(ctx):
        for j in range(T):
            cache[2][b, g, c + j, j % D] = 0xff if j % 2 else 0x7f
            want[b, j:, g * G:, j % D] = True
    note(f"verify q8 NaN in every draft row, T={T} D={D} P={P}")
    out, mass, lse = run_verify(q, cache, ctx, P=P, seed=3)
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(out[~want], clean[0][~want])
    assert torch.equal(mass, clean[1]) and torch.equal(lse, clean[2])
