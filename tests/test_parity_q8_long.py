"""GPU parity of the 8-bit verify where a lost or doubled token has to show: inputs and bounds of ``attn_bounds``,
which ``test_attn_bounds`` shows to refuse a lost block, a lost unit, a token read twice and a result of zeros."""
import pytest
import torch

import attn_bounds as A
from gpu_util import note
from test_parity_q8 import run_verify

pytestmark = pytest.mark.gpu

CASES = [
    # B, T, Hq, Hkv, D, contexts, P, mass
    (1, 17, 16, 2, 128, [131072 - 17], 0, True),
    (1, 1, 16, 2, 128, [131071], 0, True),
    (1, 1, 16, 2, 128, [131071], 64, False),
    (1, 9, 64, 8, 128, [12800], 32, True),
    (1, 6, 28, 4, 128, [6432], 0, True),
    (4, 9, 40, 8, 128, [16384, 33280, 20001, 16500], 32, True),
    (16, 1, 28, 4, 128, [2048 + 953 * i for i in range(16)], 64, False),
    (2, 32, 20, 1, 64, [9000, 4097], 0, True),
    (1, 5, 4, 1, 64, [40000], 256, True),
    (3, 1, 64, 64, 64, [20000, 0, 6000], 32, True),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[0]}T{c[1]}H{c[2]}/{c[3]}D{c[4]}c{c[5][0]}P{c[6]}")
def test_every_token_counts_once(case):
    B, T, Hq, Hkv, D, ctx, P, mass = case
    rows = -(-(max(ctx) + T) // 32) * 32
    q, cache, scale = A.aimed(B, T, Hq, Hkv, D, rows, "cuda")
    note(f"verify q8, every token counts {case}")
    out, m, lse = run_verify(q, cache, ctx, scale=scale, P=P, seed=B, want_mass=mass)
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    (ro, rl, rm), (bo, bl, bm) = A.reference(q, A.values(*cache[:2]), A.values(*cache[2:]), ctx, scale, cus)
    for name, got, want, bound in (("out", out, ro, bo), ("lse", lse, rl, bl)) + ((("mass", m[:, :rows], rm, bm),) if mass else ()):
        off = ((got.double() - want).abs() / bound.clamp_min(1e-300)).max().item()
        print(f"[bounds] {name}: at most {off:.3f} of the bound", flush=True)
        assert not A.beyond(got, want, bound), name
    if mass:
        for b, c in enumerate(ctx):
            assert not m[b, c + T:].any()


@pytest.mark.parametrize("T", [1, 17])
def test_random_rows_of_a_long_cache_within_the_tight_bounds(T):
    g = torch.Generator(device="cuda")
    g.manual_seed(40 + T)
    Hq, Hkv, D, ctx = 16, 2, 128, 131072 - T
    codes = [torch.randn((1, Hkv, 131072, D), device="cuda", generator=g).to(torch.float8_e4m3fn).view(torch.uint8)
             for _ in range(2)]
    exps = [torch.randint(125, 128, (1, Hkv, 131072), device="cuda", generator=g, dtype=torch.uint8) for _ in range(2)]
    cache = (codes[0], exps[0], codes[1], exps[1])
    q = torch.randn((1, T, Hq, D), device="cuda", generator=g).bfloat16()
    note(f"verify q8, 131072 random rows, T = {T}")
    out, m, lse = run_verify(q, cache, [ctx])
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    (ro, rl, rm), (bo, bl, bm) = A.reference(q, A.values(*cache[:2]), A.values(*cache[2:]), [ctx], D ** -0.5, cus)
    for name, got, want, bound in (("out", out, ro, bo), ("lse", lse, rl, bl), ("mass", m, rm, bm)):
        off = ((got.double() - want).abs() / bound.clamp_min(1e-300)).max().item()
        print(f"[bounds] {name}: at most {off:.3f} of the bound", flush=True)
        assert not A.beyond(got, want, bound), name
