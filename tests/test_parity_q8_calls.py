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
