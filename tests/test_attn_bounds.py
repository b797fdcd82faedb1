"""What the bounds of ``attn_bounds`` refuse and what they allow, on the CPU (not gpu)."""
import pytest
import torch

import attn_bounds as A

CASES = [
    # T, G, D, context
    (17, 8, 128, 131072 - 17), (1, 8, 128, 131071), (1, 7, 128, 16383), (9, 8, 128, 12800), (5, 4, 64, 40000),
]


def attention(q, K, V, ctx, scale, weight):
    """out, lse, mass of one sequence and KV head, a token counting ``weight`` times (0: lost, 2: read twice)."""
    _, T, G, D = q.shape
    n = ctx + T
    s = scale * q[0].double().reshape(T * G, D) @ K[0, 0, :n].t()
    s = s.masked_fill(torch.arange(n)[None] > ctx + torch.arange(T).repeat_interleave(G)[:, None], -torch.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - top) * weight[:n]
    z = p.sum(dim=-1, keepdim=True)
    out = (p @ V[0, 0, :n] / z).view(1, T, G, D)
    return out, (top + z.log()).view(T, G).t()[None], (p / z).sum(dim=0)[None]


@pytest.mark.parametrize("T,G,D,ctx", CASES)
def test_a_lost_block_a_token_read_twice_and_zeros_are_refused(T, G, D, ctx):
    rows = -(-(ctx + T) // 32) * 32
    q, c, scale = A.aimed(1, T, G, 1, D, rows)
    K, V = A.values(*c[:2]), A.values(*c[2:])
    (o, l, m), (bo, bl, bm) = A.reference(q, K, V, [ctx], scale)
    one = torch.ones(rows, dtype=torch.float64)
    got = attention(q, K, V, ctx, scale, one)
    assert not A.beyond(got[0], o, bo) and not A.beyond(got[1], l, bl)
    assert not A.beyond(got[2], m[:, :ctx + T], bm[:, :ctx + T])
    assert A.beyond(torch.zeros_like(o), o, bo) and A.beyond(torch.zeros_like(m), m, bm)
    last = (ctx // 64 - 1) * 64
    for first in (0, 64, last // 128 * 64, last):
        for size in (64, 32):                       # a block, a unit: lost, read twice
            for times in (0.0, 2.0):
                w = one.clone()
                w[first:first + size] = times
                out, lse, mass = attention(q, K, V, ctx, scale, w)
                assert A.beyond(lse, l, bl), (first, size, times)
                if size == 64:
                    assert A.beyond(out, o, bo), (first, times)
                assert A.beyond(mass, m[:, :ctx + T], bm[:, :ctx + T]), (first, size, times)
        if T * G >= 32:                             # one token, at which one class of rows looks
            w = one.clone()
            w[first + 5] = 0.0
            assert A.beyond(attention(q, K, V, ctx, scale, w)[0], o, bo), first


def test_values_of_another_block_and_a_rows_wrong_exponent_are_refused():
    T, G, D, ctx = 9, 8, 128, 6400
    q, c, scale = A.aimed(1, T, G, 1, D, 6432)
    K, V = A.values(*c[:2]), A.values(*c[2:])
    (o, _, _), (bo, _, _) = A.reference(q, K, V, [ctx], scale)
    one = torch.ones(6432, dtype=torch.float64)
    W = V.clone()
    W[0, 0, 640:704] = V[0, 0, 704:768]
    assert A.beyond(attention(q, K, W, ctx, scale, one)[0], o, bo)
    exps = c[3].clone()
    exps[0, 0, 1000:1032] = c[3][0, 0, 1001:1033]
    W = A.values(c[2], exps)
    assert A.beyond(attention(q, K, W, ctx, scale, one)[0], o, bo)


@pytest.mark.parametrize("T,G,D,ctx", CASES[2:])
def test_the_kernels_roundings_are_allowed(T, G, D, ctx):
    """fp32 sums and probabilities rounded to bf16, over random rows."""
    g = torch.Generator().manual_seed(ctx)
    n = ctx + T
    K, V = (torch.randn((1, 1, n, D), generator=g).to(torch.float8_e4m3fn).double() for _ in range(2))
    q = torch.randn((1, T, G, D), generator=g).bfloat16()
    (o, l, m), (bo, bl, bm) = A.reference(q, K, V, [ctx], D ** -0.5)
    s = D ** -0.5 * q[0].float().reshape(T * G, D) @ K[0, 0].float().t()
    s = s.masked_fill(torch.arange(n)[None] > ctx + torch.arange(T).repeat_interleave(G)[:, None], -torch.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - top)
    z = p.double().sum(dim=-1, keepdim=True).float()
    r = p.bfloat16().float()
    out = ((r @ V[0, 0].float()) / r.double().sum(dim=-1, keepdim=True).float()).bfloat16().view(1, T, G, D)
    assert not A.beyond(out, o, bo)
    assert not A.beyond((top + z.log()).view(T, G).t()[None], l, bl)
    assert not A.beyond((p / z).sum(dim=0)[None], m, bm)
