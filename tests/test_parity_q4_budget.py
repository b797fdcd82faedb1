"""GPU parity of the 4-bit verify where a KV head has more sets of row tiles than its stream
has compute units: workgroups take several sets, one after the other."""
import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
from gpu_util import note
from test_parity_q4 import check_all, i32, random_cache
from test_parity_q4_ragged import check_ragged, dirty
from test_parity_q8 import queries, status_word

pytestmark = pytest.mark.gpu


@pytest.fixture
def small_stream():
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    pv.set_stream_cu_budget(s, 8)
    yield s
    torch.cuda.synchronize()
    pv.set_stream_cu_budget(s, 0)


def on(stream, f):
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        got = f()
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("B,Hkv,G,D,ctx", [
    (1, 1, 20, 64, [900]), (1, 1, 20, 128, [333]),               # 14 sets; the workgroups write the results
    (1, 1, 20, 128, [5000]), (2, 1, 20, 64, [3000, 70]),         # one share, combined; of two sequences
    (1, 2, 15, 64, [800]), (2, 3, 13, 128, [100, 1200]),         # pieces of several KV heads; 10 and 9 sets
])
def test_more_sets_than_compute_units(small_stream, B, Hkv, G, D, ctx):
    rng = np.random.default_rng(G + D + sum(ctx))
    T = 32
    q, cache = queries(rng, B, T, G * Hkv, D), random_cache(rng, B, Hkv, max(ctx) + T, D)
    st = status_word()
    note(f"verify q4 on 8 compute units, B{B} H{G * Hkv}/{Hkv} D{D} {ctx}")
    got = on(small_stream, lambda: pv.verify_attn_q4(q, *cache, i32(ctx), max_ctx=max(ctx), status=st))
    check_all(got, q, cache, ctx)
    out, none, lse = on(small_stream, lambda: pv.verify_attn_q4(q, *cache, i32(ctx), max_ctx=max(ctx), want_mass=False,
                                                                status=st))
    assert none is None and torch.equal(out, got[0]) and torch.equal(lse, got[2])
    # a NaN in the values of a new row: every later row sees it, in every set
    bad = [t.clone() for t in cache]
    want = torch.zeros_like(out, dtype=torch.bool)
    for b, c in enumerate(ctx):
        bad[3][b, Hkv - 1, c + 2 + b, 1] = 255
        want[b, 2 + b:, -G:, 32:64] = True
    note("the same with NaN values")
    out, _, lse = on(small_stream, lambda: pv.verify_attn_q4(q, *bad, i32(ctx), max_ctx=max(ctx), status=st))
    assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], got[0][~want]) and torch.equal(lse, got[2])
    # sequences with their own numbers of rows
    new = [T - 9, 1][:B]
    qd, cd = dirty(q, cache, ctx, new, 255)
    note(f"the same with {new} rows")
    ragged = on(small_stream, lambda: pv.verify_attn_q4(qd, *cd, i32(ctx), n_new=i32(new), max_ctx=max(ctx), status=st))
    check_ragged(ragged, q, cache, ctx, new)
    assert int(st.item()) == 0
