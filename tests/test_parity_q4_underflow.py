"""GPU parity of the 4-bit verify where a row's largest probability exceeds others by almost
the whole range of its sums: these still decide the columns in which its value is 0."""
import numpy as np
import pytest
import torch

import paper_2603_19610_amd as pv
from gpu_util import note
from test_parity_q4 import i32, to_cache
from test_parity_q8 import cap32, status_word

pytestmark = pytest.mark.gpu


def scores_to_keys(x, scores):
    """Rows whose product with a query of ones is the score: multiples of 4 up to 128 in channels that hold them exactly."""
    for t, s in scores.items():
        x[t, 0], x[t, 32] = s // 32 * 32, s % 32
    assert all(s % 32 in (0, 4, 8, 12, 16, 24) and s // 32 in (0, 1, 2, 3, 4) for s in scores.values())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,top,cus", [
    (800, 512, 0),      # the workgroup's waves take units in turn: the wave of the small ones
    (800, 544, 0),      # another wave
    (20000, 512, 0), (20000, 544, 0), (20000, 19000, 0), (20000, 3000, 0),      # shares of few units
    (20000, 512, 8), (20000, 544, 8), (20000, 19000, 8), (20000, 3000, 8),      # of many: the same, and another share
])
def test_probabilities_far_below_the_largest(D, n, top, cus):
    """Scores (in log2) 0, but 24 at two tokens of unit 8, which raises no reference, and 128 at `top`.  Probabilities are
    exact powers of two; values are 0 at the top and 1 and 0.5 at the two in column 0: 1.5 * 2^-104 there, for which all
    n tokens of score 0 (2^-128 each, values 0 but at token 3) are nothing.  Column 1 is the top's own value.  The quotient
    and its conversion are rounded: 2^-8, and each change of a reference by a power of two is off by a few units of 2^-23."""
    x, v = np.zeros((cap32(n), D)), np.zeros((cap32(n), D))
    scores_to_keys(x, {256: 24, 270: 24, top: 128})
    v[256, 0], v[270, 0], v[top, 1] = 1.0, 0.5, 3.0
    cache = [dev[None, None] for dev in (*to_cache(x), *to_cache(v))]
    q = torch.ones((1, 1, 1, D), dtype=torch.bfloat16, device="cuda")
    st, at, stream = status_word(), i32([n - 1]), torch.cuda.Stream()
    note(f"verify q4 probabilities of 2^-104, D{D} {n} tokens, the largest at {top}, {cus} compute units")
    torch.cuda.synchronize()
    pv.set_stream_cu_budget(stream, cus)
    try:
        with torch.cuda.stream(stream):
            out, mass, lse = pv.verify_attn_q4(q, *cache, at, scale=float(np.log(2.0)), status=st)
        torch.cuda.synchronize()
    finally:
        pv.set_stream_cu_budget(stream, 0)
    assert int(st.item()) == 0
    want = 1.5 * 2.0 ** -104
    assert abs(out[0, 0, 0, 0].item() / want - 1) <= 2.0 ** -8 + 2.0 ** -18
    assert out[0, 0, 0, 1].item() == 3.0 and not out[0, 0, 0, 2:].any()
    assert abs(mass[0, 256].item() * 2.0 ** 104 - 1) <= 2.0 ** -16 and abs(lse.item() / (128 * np.log(2.0)) - 1) <= 2.0 ** -22


def test_sums_of_many_small_ones_far_below_the_largest():
    """A whole unit of every wave at 24, over 100000 tokens, 128 at the last: their sum is what column 0 is."""
    n, D = 100000, 64
    x, v = np.zeros((cap32(n), D)), np.zeros((cap32(n), D))
    scores_to_keys(x, {n - 1: 128})
    x[256:n - 1, 32] = 24.0
    v[:n - 1, 0] = 1.0
    cache = [dev[None, None] for dev in (*to_cache(x), *to_cache(v))]
    q = torch.ones((1, 1, 1, D), dtype=torch.bfloat16, device="cuda")
    note("verify q4 99743 probabilities of 2^-104")
    out, mass, lse = pv.verify_attn_q4(q, *cache, i32([n - 1]), scale=float(np.log(2.0)))
    want = (n - 1 - 256) * 2.0 ** -104
    assert abs(out[0, 0, 0, 0].item() / want - 1) <= 2.0 ** -8 + n * 2.0 ** -24
