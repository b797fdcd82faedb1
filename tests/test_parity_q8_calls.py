"""GPU parity of the 8-bit calls in the ways that programs make them: captured
graphs beside each other, prompts, calls without mass or log-sum-exp, 32-bit
sources.  Reference and bounds are those of ``test_parity_q8``."""
import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
from gpu_util import note
from test_parity_q8 import queries, random_cache

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
