"""Page tables, rotary rows by slot and the 4-bit key-value cache: their calls, and what those calls compute.

Five kinds of case:

* ``pages``     a batch's page tables grown for its new rows, the slots of those
                rows, and the tables cut back to the rows that stay.
* ``rotary``    rotary embedding of rows (both pairings, part of a head, scaled
                frequencies) and the append of their keys and values by slot.
* ``append``    the same into a 4-bit cache; the rows are read back as values.
* ``handover``  a prefill's cache of all layers into a 4-bit one, and the draft's
                compact cache of its kept rows, as values.
* ``verify``    attention of T new rows over a 4-bit cache with every token's
                attention mass; T = 1 without mass is a decode step.

A 4-bit row of D values is, for every 32 of them, e2m1 codes (0, 0.5, 1, 1.5, 2,
3, 4, 6 and a sign) and one exponent byte e: a value is ``code * 2**(e - 127)``,
e the smallest number in [1, 254] that keeps the block's largest magnitude
within 7.  Two codes share a byte, the first in its low half.  A padded cache is
[B][Hkv][n_cap][D / 2] with exponents [B][Hkv][n_cap][D / 32]; a paged one
[n_pages][Hkv][page][...].

Shapes are those of ``workloads`` (LLaVA-OV 7B and 72B, Qwen2.5-VL-32B, the
131K-token video); ``draw`` spreads over the ranges around them.
"""
import math
import random

import torch

own = False

BF16, F32 = "bf16", "f32"
_BASE = 1.0e6


# ------------------------------------------------------------------ cases --
def _named(name, case):
    return dict(case, name=name) if name else case


def _pages(name, B, page, ctx_lo, ctx_hi, T, admit=False):
    return _named(name, dict(kind="pages", B=B, page=page, ctx_lo=ctx_lo, ctx_hi=ctx_hi, T=T, admit=admit))


def _rotary(name, kind, dtype, B, T, hq, hkv, D, ctx_lo, ctx_hi, page=0, rot=0, inter=False, scaling="",
            mrope=False):
    return _named(name, dict(kind=kind, dtype=dtype, B=B, T=T, hq=hq, hkv=hkv, D=D, ctx_lo=ctx_lo,
                             ctx_hi=ctx_hi, page=page, rot=rot or D, inter=inter, scaling=scaling,
                             mrope=mrope))


def _handover(name, dtype, to, layers, B, hkv, D, m_lo, m_hi, n, keep_num, keep_den, page=0):
    return _named(name, dict(kind="handover", dtype=dtype, to=to, layers=layers, B=B, hkv=hkv, D=D, m_lo=m_lo,
                             m_hi=m_hi, n=n, keep_num=keep_num, keep_den=keep_den, page=page))


def _verify(name, B, T, hq, hkv, D, ctx_lo, ctx_hi, page=0, mass=True):
    return _named(name, dict(kind="verify", B=B, T=T, hq=hq, hkv=hkv, D=D, ctx_lo=ctx_lo, ctx_hi=ctx_hi,
                             page=page, mass=mass))


def listed():
    return [
        # A serving batch's verify step: up to nine rows for each of 64 sequences, all but
        # the accepted ones given back.  All latency.
        _pages("pages-verify", 64, 32, 2048, 33280, 9),
        # Sixteen long prompts admitted, their rows' slots, and (a cancelled batch) all pages given back.
        _pages("pages-admit", 16, 32, 0, 0, 33280, admit=True),
        # The 7B target's six verify rows into a padded cache: a small call, all latency.
        _rotary("rotary-7b", "rotary", BF16, 1, 6, 28, 4, 128, 6432, 6432),
        # A whole prompt of the 72B shape, half of every head rotated in adjacent pairs,
        # frequencies scaled to a context four times as long.
        _rotary("rotary-72b-prompt", "rotary", BF16, 1, 12800, 64, 8, 128, 0, 0, page=64, rot=64, inter=True,
                scaling="yarn"),
        # One token of each of sixteen 7B sequences into a paged 4-bit cache.
        _rotary("append-batch", "append", BF16, 16, 1, 28, 4, 128, 2048, 16384, page=64),
        # The 72B target's whole prompt, one layer of its prefill, into a 4-bit cache.
        _rotary("append-72b-prompt", "append", BF16, 1, 12800, 64, 8, 128, 0, 0),
        # One layer of the 7B draft's own compact cache, made in bf16, handed on in 4 bits.
        _handover("handover-draft-7b", BF16, BF16, 1, 1, 4, 128, 627, 627, 160, 1, 2),
        # The 7B target's cache of all 28 layers after its prefill, and its draft's tenth of it.
        _handover("handover-7b", BF16, BF16, 28, 1, 4, 128, 6272, 6272, 160, 1, 10),
        # The 7B draft's decode step over its compact cache: one row, no mass.  All latency.
        _verify("decode-draft-7b", 1, 1, 28, 4, 128, 787, 787, mass=False),
        # One token of each of sixteen 7B sequences, ragged, paged: batched decoding.
        _verify("decode-batch-paged", 16, 1, 28, 4, 128, 2048, 16384, page=64, mass=False),
        # A layer of the 72B target's verify forward, 64 frames, nine rows.
        _verify("verify-72b", 1, 9, 64, 8, 128, 12800, 12800),
        # One layer over a 131K-token video, seventeen rows: the longest context.
        _verify("verify-long", 1, 17, 64, 8, 128, 132096, 132096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pages", "rotary", "append", "handover", "verify", "verify", "verify", "verify"])
    hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 4, 5, 7, 8])
    D = rng.choice([64, 128, 128])
    page = rng.choice([0, 0, 32, 64, 256])
    B = rng.choice([1, 1, 2, 3, 4])
    if kind == "pages":
        page = rng.choice([32, 64, 256])
        if rng.random() < 0.3:
            B = rng.randint(1, 16)
            return _pages(None, B, page, 0, 0, _log(rng, 1, 33280), admit=True)
        B, hi = _log(rng, 1, 256), _log(rng, 1, 33280)
        return _pages(None, B, page, rng.randint(hi // 3, hi), hi, rng.randint(1, 32))
    if kind in ("rotary", "append"):
        T = rng.choice([rng.randint(1, 32), _log(rng, 1, 12800 // B)])
        B = rng.choice([B, rng.randint(1, 16)]) if T == 1 else B
        ctx = _log(rng, 1, 30000)
        mrope = rng.random() < 0.3
        dtype = BF16 if kind == "append" or 8 * group * hkv * T * B > 400000 else rng.choice([BF16, F32])
        return _rotary(None, kind, dtype, B, T, group * hkv, hkv, D, rng.randint(0, ctx), ctx, page=page,
                       rot=rng.choice([D, D, D // 2, D // 4]), inter=rng.random() < 0.4,
                       scaling=rng.choice(["", "linear", "parts", "yarn"]), mrope=mrope)
    if kind == "verify":
        T = rng.choice([1, 1, rng.randint(2, 9), rng.randint(2, 17), rng.randint(2, 32)])
        B = rng.choice([B, rng.randint(1, 16)]) if T == 1 else B
        # at most the work of the longest listed one
        hi = _log(rng, 1, 132096 * min(1, 17 * 64 * 128 / (T * group * hkv * D)) / B)
        return _verify(None, B, T, group * hkv, hkv, D, rng.randint(hi // 3, hi), hi, page=page,
                       mass=T > 1 or rng.random() < 0.3)
    dtype, to, hi = rng.choice([BF16, BF16, F32]), rng.choice([BF16, BF16, F32]), _log(rng, 20, 40000 // B)
    c = _handover(None, dtype, to, 1, B, hkv, D, rng.randint(hi // 2, hi), hi, rng.randint(1, 1024),
                  rng.randint(1, 50), 100, page=page)
    layers = rng.choice([1, 28, 64, 80])
    return dict(c, layers=max(1, min(layers, int(450e6 / work(c)["bytes"]))))


# ----------------------------------------------------------------- inputs --
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 41)
    return g


def _lengths(lo, hi, B):
    """Lengths of a ragged batch: the longest is hi, the others between."""
    r = random.Random(7919 * lo + 31 * hi + B)
    return [hi] + [r.randint(lo, hi) for _ in range(B - 1)]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cap(rows):
    """Row capacity of a padded cache: a multiple of 32."""
    return max(32, -(-rows // 32) * 32)


def _power(e):
    """2**(e - 127) for whole numbers e in [1, 254]."""
    return torch.bitwise_left_shift(e.int(), 23).view(torch.float32)


def _codes4(x):
    """e2m1 codes (whole numbers 0 .. 15) and exponents of the 32-blocks of the rows of x."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(dim=-1).view(torch.int32)
    # top = 2**(b - 127) * 1.m for its exponent b and mantissa m; 7 = 2**2 * 1.75
    e = ((top >> 23) - 2 + ((top & 0x7fffff) > 0x600000)).clamp(1, 254)
    x = x * _power(254 - e)[..., None]
    a = x.abs()
    c = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return (c + 8 * torch.signbit(x)).flatten(-2), e


def _to_4bit(x):
    """Packed codes and exponents of the rows of x."""
    c, e = _codes4(x)
    c = c.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4), e.to(torch.uint8)


def _table():
    v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float32, device="cuda")
    return torch.cat([v, -v])


def _held(x):
    """The values that the 4-bit rows of x stand for."""
    c, e = _codes4(x)
    return (_table()[c].unflatten(-1, (-1, 32)) * _power(e)[..., None]).flatten(-2)


def _unpack(codes, exps):
    """The values of packed rows, in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    return (_table()[c].unflatten(-1, (-1, 32)) * _power(exps)[..., None]).flatten(-2)


def _rows(g, shape):
    """Keys or values of one layer as a model has them: channels of different
    size, a few rows much larger or smaller than the rest."""
    x = torch.randn(shape, device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn(shape[-1:], device="cuda", generator=g))
    size = torch.exp(0.4 * torch.randn(shape[:-1] + (1,), device="cuda", generator=g))
    return x * size


def _page_table(g, case, lens):
    """A page table for rows 0 .. lens[b] - 1, and the pool's size (a padded cache: None, B)."""
    B, P = case["B"], case["page"]
    if not P:
        return None, B
    need = [-(-n // P) for n in lens]
    n_pages = sum(need) + 3
    perm = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
    o = 0
    for b in range(B):
        table[b, :need[b]] = perm[o:o + need[b]]
        o += need[b]
    return table, n_pages


def _cache4(g, case, lens, layers=None):
    """A 4-bit cache of rows 0 .. lens[b] - 1; rows past them hold arbitrary codes."""
    hkv, D = case["hkv"], case["D"]
    table, n0 = _page_table(g, case, lens)
    shape = (n0, hkv, case["page"] or _cap(max(lens)), D)
    out = []
    for _ in range(2):
        parts = [_to_4bit(_rows(g, shape)) for _ in range(layers or 1)]
        out += [torch.stack(x) for x in zip(*parts)] if layers else list(parts[0])
    return dict(kc=out[0], ke=out[1], vc=out[2], ve=out[3], table=table)


def _at(s, b, rows):
    """Where rows (same shape as b) of sequences b lie in a cache: the indices before and after the head's."""
    if s["table"] is None:
        return b, rows
    P = s["block"]
    return s["table"][b, rows // P].long(), rows % P


def _prepare_pages(case, seed):
    g = _gen(seed)
    B, P, T = case["B"], case["page"], case["T"]
    r = random.Random(int(seed))
    ctx = _lengths(case["ctx_lo"], case["ctx_hi"], B)
    new = [T] + [r.randint(max(1, T // 2), T) if case["admit"] else r.randint(1, T) for _ in range(B - 1)]
    stay = [0 if case["admit"] else c + r.randint(1, n) for c, n in zip(ctx, new)]
    # the table holds the context's pages; the pool has room for the batch and some to spare
    held = [-(-c // P) for c in ctx]
    most = -(-(max(ctx) + T) // P)
    n_pages = sum(-(-(c + T) // P) for c in ctx) + 16
    spare = n_pages - sum(held)
    perm = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((B, most), -1, dtype=torch.int32, device="cuda")
    o = 0
    for b in range(B):
        table[b, :held[b]] = perm[o:o + held[b]]
        o += held[b]
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:spare] = perm[o:]
    return dict(B=B, P=P, table=table, free=free, n_free=_i32([spare]), held=_i32(held), ctx=_i32(ctx), new=_i32(new),
                want=_i32([c + n for c, n in zip(ctx, new)]), stay=_i32(stay), rows=B * T)


_SCALED = {"": dict(), "linear": dict(factor=4.0), "parts": dict(factor=8.0, orig_ctx=8192.0, alpha=1.0, beta=4.0),
           "yarn": dict(factor=4.0, orig_ctx=32768.0, alpha=1.0, beta=32.0, mscale=1.1386)}


def _prepare_rotary(case, seed):
    g = _gen(seed)
    B, T, hq, hkv, D, R = (case[k] for k in ("B", "T", "hq", "hkv", "D", "rot"))
    lens = _lengths(case["ctx_lo"], case["ctx_hi"], B)
    full = [n + T for n in lens]
    ctx = _i32(lens)
    block = case["page"] or _cap(max(full))
    dt = torch.bfloat16 if case["dtype"] == BF16 else torch.float32
    if case["kind"] == "append":
        s = _cache4(g, case, full)
    else:
        table, n0 = _page_table(g, case, full)
        s = dict(table=table, k=_rows(g, (n0, hkv, block, D)).to(dt), v=_rows(g, (n0, hkv, block, D)).to(dt))
    s = dict(s, ctx=ctx, block=block, T=T)
    row = ctx[:, None].long() + torch.arange(T, device="cuda")
    at, r = _at(s, torch.arange(B, device="cuda")[:, None].expand(B, T), row)
    s["slots"] = (at * block + r).reshape(-1)
    pos = row.reshape(-1).to(torch.int32)
    rot = dict(rot_dim=R, base=_BASE, layout="interleaved" if case["inter"] else "half")
    if case["scaling"]:
        rot = dict(rot, scaling=case["scaling"], **_SCALED[case["scaling"]])
    if case["mrope"]:
        lag = torch.randint(0, 64, (2, B * T), device="cuda", generator=g, dtype=torch.int32)
        pos = torch.cat([pos[None], torch.relu(pos[None] - lag)]).contiguous()
        rot["sections"] = (R // 8, R // 4 - R // 16, R // 4 - R // 16)
    # queries, keys and values are slices of the rows of one projection
    qkv = _rows(g, (B * T, hq + 2 * hkv, D)).to(dt)
    return dict(s, pos=pos, rot=rot, q=qkv[:, :hq], k_new=qkv[:, hq:hq + hkv], v_new=qkv[:, hq + hkv:],
                n_new=_i32([T] * B), none=_i32([0] * B))


def _prepare_handover(case, seed):
    g = _gen(seed)
    L, B, hkv, D, n = (case[k] for k in ("layers", "B", "hkv", "D", "n"))
    m = _lengths(case["m_lo"], case["m_hi"], B)
    lens = [x + n for x in m]
    keep = [x * case["keep_num"] // case["keep_den"] for x in m]
    k_cap = max(1, max(keep))
    idx = torch.full((B, k_cap), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        at = torch.randperm(m[b], device="cuda", generator=g)[:keep[b]].sort().values
        idx[b, :keep[b]] = at.to(torch.int32)
    table, n0 = _page_table(g, case, lens)
    block = case["page"] or _cap(max(lens))
    shape = (L, n0, hkv, block)
    cache = [torch.zeros(shape + (w,), dtype=torch.uint8, device="cuda") for w in (D // 2, D // 32) * 2]
    dt = torch.bfloat16 if case["dtype"] == BF16 else torch.float32
    cap = max(lens) + 5     # the prefill's own capacity
    src = [torch.stack([_rows(g, (B, hkv, cap, D)).to(dt) for _ in range(L)]) for _ in range(2)]
    return dict(k=src[0], v=src[1], lens=_i32(lens), cache=cache, table=table, block=block, idx=idx, keep=_i32(keep),
                m=_i32(m), tail=_i32([n] * B), dst_cap=max(keep) + n,
                to=torch.bfloat16 if case["to"] == BF16 else torch.float32)


def _prepare_verify(case, seed):
    g = _gen(seed)
    B, T, hq, hkv, D = (case[k] for k in ("B", "T", "hq", "hkv", "D"))
    lens = _lengths(case["ctx_lo"], case["ctx_hi"], B)
    s = _cache4(g, case, [n + T for n in lens])
    s["block"] = case["page"]
    # queries whose scores are as wide as a model's, and, as a model's do, look
    # much at the first rows and at one row in fifty
    q = torch.randn((B, T, hq, D), device="cuda", generator=g)
    mean_q = q.view(B, T, hkv, hq // hkv, D).mean(dim=(1, 3))
    mean_q = 3.0 * mean_q / mean_q.norm(dim=-1, keepdim=True)
    for b, n in enumerate(lens):
        at = torch.randint(0, n + T, (max(1, (n + T) // 50),), device="cuda", generator=g)
        at = torch.cat([at, torch.zeros(1, dtype=at.dtype, device="cuda")]).unique()
        codes, exps = _to_4bit(torch.randn((at.numel(), hkv, D), device="cuda", generator=g) + mean_q[b][None])
        i, r = _at(s, torch.full_like(at, b), at)
        s["kc"][i, :, r] = codes
        s["ke"][i, :, r] = exps
    return dict(s, q=q.bfloat16(), ctx=_i32(lens), max_ctx=max(lens), mass=case["mass"])


def prepare(case, seed):
    s = {"pages": _prepare_pages, "rotary": _prepare_rotary, "append": _prepare_rotary,
         "handover": _prepare_handover, "verify": _prepare_verify}[case["kind"]](case, seed)
    return dict(s, kind=case["kind"])


# ------------------------------------------------------- the plain forms --
def _resize(s, rows):
    """The tables for `rows` of each sequence: pages that are too many back on
    the stack, then those that are missing off its top, in order."""
    B, P = s["B"], s["P"]
    table, free, held = s["table"], s["free"], s["held"].long()
    need = (rows.long() + P - 1) // P
    col = torch.arange(table.shape[1], device="cuda")[None]
    back = (col >= need[:, None]) & (col < held[:, None])
    top = s["n_free"].long()
    # (entries that stay go to a place past the stack)
    where = torch.where(back, top + torch.cumsum(back.flatten().long(), 0).view_as(table) - 1, free.numel())
    stack = torch.cat([free, free[:1]]).scatter_(0, where.flatten(), table.flatten())[:-1]
    table.masked_fill_(back, -1)
    top = top + back.sum()
    more = (need - held).clamp_min(0)
    upto = torch.cumsum(more, 0)
    fits = upto <= top
    take = torch.where(fits, more, torch.zeros_like(more))
    first = upto - more
    now = (col >= held[:, None]) & (col < (held + take)[:, None])
    nth = (first - held)[:, None] + col
    table.copy_(torch.where(now, stack[(top - 1 - nth).clamp(0, free.numel() - 1)], table))
    free.copy_(stack)
    s["held"].copy_(torch.minimum(held, need) + take)
    s["n_free"].copy_(top - take.sum())
    return (take == more).to(torch.int32)


def _plain_pages(s):
    B, P = s["B"], s["P"]
    granted = _resize(s, s["want"])
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.cumsum(s["new"].long(), 0)])
    i = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(start, i, right=True) - 1
    real = seq < B
    b = seq.clamp_max(B - 1)
    row = s["ctx"].long()[b] + i - start[b]
    page = s["table"][b, (row // P).clamp_max(s["table"].shape[1] - 1)].long()
    out = dict(slots=torch.where(real, page * P + row % P, -1), pos=torch.where(real, row, 0).to(torch.int32),
               seq=torch.where(real, b, -1).to(torch.int32), start=start.to(torch.int32))
    kept = _resize(s, s["stay"])
    top = torch.arange(s["free"].numel(), device="cuda") < s["n_free"]
    return dict(out, granted=granted, kept=kept, table=s["table"], held=s["held"], n_free=s["n_free"],
                free=torch.where(top, s["free"], -1))


def _frequencies(rot):
    R = rot["rot_dim"]
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    f = torch.exp(i * (-2.0 / R * math.log(rot["base"])))
    kind, s = rot.get("scaling"), rot.get("factor", 1.0)
    if kind == "linear":
        return f / s
    if kind == "parts":
        turns = rot["orig_ctx"] * f / (2 * math.pi)
        w = ((turns - rot["alpha"]) / (rot["beta"] - rot["alpha"])).clamp(0, 1)
        return f * (w + (1 - w) / s)
    if kind == "yarn":
        lo, hi = [R / 2 * math.log(rot["orig_ctx"] / (2 * math.pi * x)) / math.log(rot["base"])
                  for x in (rot["beta"], rot["alpha"])]
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), R - 1)
        w = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (w + (1 - w) / s)
    return f


def _rotate(s, x):
    """Rows x [N][H][D] turned by their positions (angles in 64 bits), in 32 bits."""
    rot, N = s["rot"], x.shape[0]
    R = rot["rot_dim"]
    h = R // 2
    if "sections" in rot:
        i = torch.arange(h, device="cuda")
        axis = (i >= rot["sections"][0]).long() + (i >= rot["sections"][0] + rot["sections"][1]).long()
        p = s["pos"].double()[axis].t()
    else:
        p = s["pos"].double()[:, None].expand(N, h)
    ang = (p * _frequencies(rot))[:, None]
    cos, sin = torch.cos(ang) * rot.get("mscale", 1.0), torch.sin(ang) * rot.get("mscale", 1.0)
    x = x.double()
    if rot["layout"] == "half":
        x1, x2 = x[..., :h], x[..., h:R]
        turned = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1)
    else:
        x1, x2 = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., R:]], dim=-1).float()


def _plain_rotary(s):
    dt = s["q"].dtype
    at, r = s["slots"] // s["block"], s["slots"] % s["block"]
    s["k"][at, :, r] = _rotate(s, s["k_new"]).to(dt)
    s["v"][at, :, r] = s["v_new"]
    return dict(q=_rotate(s, s["q"]).to(dt), k=s["k"], v=s["v"])


def _plain_append(s):
    B, T = s["ctx"].numel(), s["T"]
    k = _held(_rotate(s, s["k_new"]).bfloat16())
    v = _held(s["v_new"])
    shape = (B, T) + k.shape[1:]
    return dict(q=_rotate(s, s["q"]).bfloat16(), k=k.view(shape).transpose(1, 2).bfloat16().contiguous(),
                v=v.view(shape).transpose(1, 2).bfloat16().contiguous())


def _plain_handover(s):
    L, B, hkv, cap, D = s["k"].shape
    b, i = torch.nonzero(torch.arange(cap, device="cuda")[None] < s["lens"][:, None], as_tuple=True)
    at, row = _at(s, b, i)
    for x, c, e in (("k", 0, 1), ("v", 2, 3)):
        codes, exps = _to_4bit(s[x][:, b, :, i])
        s["cache"][c][:, at, :, row] = codes
        s["cache"][e][:, at, :, row] = exps
    r = torch.arange(s["dst_cap"], device="cuda")[None]
    kept = r < s["keep"][:, None]
    b, i = torch.nonzero(r < (s["keep"] + s["tail"])[:, None], as_tuple=True)
    first = s["idx"].long().gather(1, r.clamp_max(s["idx"].shape[1] - 1).expand(B, s["dst_cap"]))
    src = torch.where(kept, first, s["m"].long()[:, None] + r - s["keep"].long()[:, None])
    at, row = _at(s, b, src[b, i])
    out = {}
    for name, c, e in (("k", 0, 1), ("v", 2, 3)):
        out[name] = torch.zeros((L, B, hkv, s["dst_cap"], D), dtype=s["to"], device="cuda")
        out[name][:, b, :, i] = _unpack(s["cache"][c][:, at, :, row], s["cache"][e][:, at, :, row]).to(s["to"])
    return out


def _values(codes, exps, table):
    """The fp32 values of a cache's rows as [B][Hkv][rows][D]."""
    if table is not None:
        at = table.clamp_min(0).long()
        codes, exps = (x[at].transpose(1, 2).flatten(2, 3) for x in (codes, exps))
    return _unpack(codes, exps)


def _plain_verify(s):
    q = s["q"].float()
    B, T, hq, D = q.shape
    hkv = s["kc"].shape[1]
    k, v = _values(s["kc"], s["ke"], s["table"]), _values(s["vc"], s["ve"], s["table"])
    rows = q.view(B, T, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, D)
    x = torch.matmul(rows, k.transpose(-1, -2)) * D ** -0.5
    n = x.shape[-1]
    last = s["ctx"].long()[:, None] + torch.arange(T, device="cuda")          # [B][T]
    hidden = torch.arange(n, device="cuda") > last[..., None]                  # [B][T][n]
    hidden = hidden[:, None, None].expand(B, hkv, hq // hkv, T, n).reshape(x.shape)
    x = x.masked_fill(hidden, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - top)
    z = p.sum(dim=-1, keepdim=True)
    p = p / z
    out = torch.matmul(p, v).view(B, hkv, hq // hkv, T, D).permute(0, 3, 1, 2, 4)
    r = dict(out=out.reshape(B, T, hq, D).bfloat16(), lse=(top + torch.log(z)).view(B, hq, T))
    if s["mass"]:
        r["mass"] = p.sum(dim=(1, 2))
    return r


# --------------------------------------------------- the framework's calls --
def _own_pages(pv, s):
    state = (s["held"], s["table"], s["free"], s["n_free"])
    granted = pv.pages_resize(s["want"], *state, page_size=s["P"])
    slots, pos, seq, start = pv.slot_map(s["ctx"], s["new"], s["rows"], page_table=s["table"], page_size=s["P"],
                                         n_pages=s["free"].numel())
    kept = pv.pages_resize(s["stay"], *state, page_size=s["P"])
    # entries of the stack past its top are not part of the answer
    top = torch.arange(s["free"].numel(), device="cuda") < s["n_free"]
    return dict(slots=slots, pos=pos, seq=seq, start=start, granted=granted, kept=kept, table=s["table"],
                held=s["held"], n_free=s["n_free"], free=torch.where(top, s["free"], -1))


def _own_run(s):
    import paper_2603_19610_amd as pv
    kind = s["kind"]
    if kind == "pages":
        return _own_pages(pv, s)
    if kind in ("rotary", "append"):
        if "plan" not in s:     # the model's rotary parameters, which a program makes once
            s["plan"] = pv.Rotary(**s["rot"])
        rows = (s["q"], s["k_new"], s["v_new"], s["pos"], s["slots"])
        if kind == "rotary":
            q = pv.rotary_append(*rows, s["k"], s["v"], rotary=s["plan"])
            return dict(q=q, k=s["k"], v=s["v"])
        cache = (s["kc"], s["ke"], s["vc"], s["ve"])
        q = pv.rotary_append_q4(*rows, *cache, rotary=s["plan"])
        sel = (s["ctx"].new_empty((s["ctx"].numel(), 0)), s["none"], s["ctx"], s["n_new"], s["T"])
        if s["table"] is None:
            k, v = pv.gather_kv_q4(*cache, *sel, dtype=torch.bfloat16)
        else:
            k, v = pv.gather_kv_q4_paged(*cache, s["table"], *sel, dtype=torch.bfloat16)
        return dict(q=q, k=k, v=v)
    table = s["table"]
    if kind == "handover":
        sel = (s["idx"], s["keep"], s["m"], s["tail"], s["dst_cap"])
        if table is None:
            pv.quantize_kv_q4(s["k"], s["v"], s["lens"], *s["cache"])
            k, v = pv.gather_kv_q4(*s["cache"], *sel, dtype=s["to"])
        else:
            pv.quantize_kv_q4_paged(s["k"], s["v"], s["lens"], *s["cache"], table)
            k, v = pv.gather_kv_q4_paged(*s["cache"], table, *sel, dtype=s["to"])
        return dict(k=k, v=v)
    cache = (s["kc"], s["ke"], s["vc"], s["ve"])
    kw = dict(max_ctx=s["max_ctx"], want_mass=s["mass"])
    if table is None:
        out, mass, lse = pv.verify_attn_q4(s["q"], *cache, s["ctx"], **kw)
    else:
        out, mass, lse = pv.verify_attn_q4_paged(s["q"], *cache, table, s["ctx"], **kw)
    return dict(out=out, lse=lse, mass=mass) if s["mass"] else dict(out=out, lse=lse)


def run(s):
    if own:
        return _own_run(s)
    return {"pages": _plain_pages, "rotary": _plain_rotary, "append": _plain_append, "handover": _plain_handover,
            "verify": _plain_verify}[s["kind"]](s)


# ------------------------------------------------------- work and accuracy --
def work(case):
    kind, B = case["kind"], case["B"]
    if kind == "pages":
        P, T = case["page"], case["T"]
        ctx = _lengths(case["ctx_lo"], case["ctx_hi"], B)
        # three quarters of an admitted prompt's most, half of a verify step's, on average
        new = 0.75 * T * B if case["admit"] else 0.5 * (T + 1) * B
        entries = 4 * (new / P if case["admit"] else B * min(1, T / P))
        return dict(bytes=16 * B * T + entries * 4 + 32 * B + 0 * sum(ctx), flops=4 * B * T)
    hkv, D = case["hkv"], case["D"]
    if kind in ("rotary", "append"):
        n, hq, size = B * case["T"], case["hq"], 2 if case["dtype"] == BF16 else 4
        kept = 2 * D * size if kind == "rotary" else 2 * (D // 2 + D // 32)
        bytes_ = n * ((2 * hq + 2 * hkv) * D * size + hkv * kept + 8 + (12 if case["mrope"] else 4))
        if kind == "append":    # read back as values
            bytes_ += n * hkv * (kept + 2 * D * 2)
        return dict(bytes=bytes_, flops=n * (3 * (hq + hkv) * case["rot"] + (4 * hkv * D if kind == "append" else 0)))
    if kind == "handover":
        m = _lengths(case["m_lo"], case["m_hi"], B)
        rows = case["layers"] * hkv * sum(x + case["n"] for x in m)
        kept = case["layers"] * hkv * sum(x * case["keep_num"] // case["keep_den"] + case["n"] for x in m)
        held = D // 2 + D // 32
        src, dst = (2 if case[k] == BF16 else 4 for k in ("dtype", "to"))
        return dict(bytes=2 * rows * (D * src + held) + 2 * kept * (held + D * dst), flops=4 * rows * D + 2 * kept * D)
    T, hq = case["T"], case["hq"]
    rows = sum(n + T for n in _lengths(case["ctx_lo"], case["ctx_hi"], B))
    size = 2 * rows * hkv * (D // 2 + D // 32) + 2 * B * T * hq * D * 2 + 4 * B * hq * T + 4 * B
    return dict(bytes=size + (4 * rows if case["mass"] else 0), flops=4 * rows * hq * T * D)


def _exact_values(x):
    """What the 4-bit rows of x stand for, in 64 bits: the nearest of the eight magnitudes."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp_min(2.0 ** -140) / 7.0)).clamp(-126, 127)
    e = torch.where(7.0 * torch.exp2(e - 1) >= top, e - 1, e)
    e = torch.where(7.0 * torch.exp2(e) < top, e + 1, e).clamp(-126, 127)
    unit = torch.exp2(e)
    a = x.abs() / unit
    out, best = torch.zeros_like(a), a.clone()
    # even codes first, so that a tie stays with them
    for m in (1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):
        d = (a - m).abs()
        closer = d < best
        out = torch.where(closer, torch.full_like(out, m), out)
        best = torch.where(closer, d, best)
    return (torch.sign(x) * out * unit).flatten(-2)


def _exact_turn(case, s):
    R, rot = case["rot"], s["rot"]
    h = R // 2
    cuts = rot.get("sections")
    pos = s["pos"].double() if cuts else s["pos"].double()[None]
    turn = torch.empty((pos.shape[1], 1, h), dtype=torch.complex128, device="cuda")
    for i in range(h):
        f = math.pow(rot["base"], -i / h)
        k = rot.get("scaling")
        near = 1.0      # how much of the unscaled frequency stays
        if k == "linear":
            near = 0.0
        elif k == "parts":
            near = (rot["orig_ctx"] * f / (2 * math.pi) - rot["alpha"]) / (rot["beta"] - rot["alpha"])
        elif k == "yarn":
            a, b = (h * math.log(rot["orig_ctx"] / (2 * math.pi * rot[x]), rot["base"]) for x in ("beta", "alpha"))
            a, b = max(math.floor(a), 0), min(math.ceil(b), R - 1)
            near = 1.0 - (i - a) / max(b - a, 0.001)
        near = min(1.0, max(0.0, near))
        f = f * near + f / rot.get("factor", 1.0) * (1.0 - near)
        axis = 0 if not cuts or i < cuts[0] else 1 if i < cuts[0] + cuts[1] else 2
        a = pos[axis] * f
        turn[:, 0, i] = torch.polar(torch.full_like(a, rot.get("mscale", 1.0)), a)

    def rotate(x):
        x = x.double()
        if case["inter"]:
            z = torch.view_as_complex(x[..., :R].unflatten(-1, (h, 2)).contiguous()) * turn
            y = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(x[..., :h].contiguous(), x[..., h:R].contiguous()) * turn
            y = torch.cat([z.real, z.imag], dim=-1)
        return torch.cat([y, x[..., R:]], dim=-1)

    return rotate


def _exact_rotary(case, seed):
    s = _prepare_rotary(case, seed)
    B, T = case["B"], case["T"]
    rotate = _exact_turn(case, s)
    q, k = rotate(s["q"]), rotate(s["k_new"])
    if case["kind"] == "append":
        # an appended key is that of a bf16 cache, in 4 bits
        k, v = _exact_values(k.to(torch.bfloat16)), _exact_values(s["v_new"])
        return dict(q=q, **{n: x.unflatten(0, (B, T)).transpose(1, 2).contiguous() for n, x in (("k", k), ("v", v))})
    out = dict(k=s["k"].double(), v=s["v"].double())
    lens = s["ctx"].tolist()
    for b in range(B):
        i = torch.arange(lens[b], lens[b] + T, device="cuda")
        for name, x in (("k", k), ("v", s["v_new"].double())):
            if case["page"]:
                out[name][s["table"][b, i // case["page"]].long(), :, i % case["page"]] = x[b * T:(b + 1) * T]
            else:
                out[name][b, :, lens[b]:lens[b] + T] = x[b * T:(b + 1) * T].transpose(0, 1)
    return dict(out, q=q)


def _exact_handover(case, seed):
    s = _prepare_handover(case, seed)
    L, B, hkv, D, n = (case[k] for k in ("layers", "B", "hkv", "D", "n"))
    out = {}
    for name in ("k", "v"):
        d = torch.zeros((L, B, hkv, s["dst_cap"], D), dtype=torch.float64, device="cuda")
        for b in range(B):
            m, keep = int(s["m"][b]), int(s["keep"][b])
            rows = torch.cat([s["idx"][b, :keep].long(), torch.arange(m, m + n, device="cuda")])
            d[:, b, :, :rows.numel()] = _exact_values(s[name][:, b][:, :, rows])
        out[name] = d
    return out


def _exact_verify(case, seed):
    s = _prepare_verify(case, seed)
    B, T, hq, hkv, D, P = (case[k] for k in ("B", "T", "hq", "hkv", "D", "page"))
    G = hq // hkv
    n_cap = s["table"].shape[1] * P if P else s["kc"].shape[2]
    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse = torch.zeros((B, T, hq, D), **f64), torch.zeros((B, hq, T), **f64)
    mass = torch.zeros((B, n_cap), **f64)
    steps = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], **f64) / 2
    for b, ctx in enumerate(s["ctx"].tolist()):
        n = ctx + T
        for h in range(hkv):
            kv = []
            for c, e in (("kc", "ke"), ("vc", "ve")):
                if P:
                    pages = s["table"][b, :-(-n // P)].long()
                    codes, exps = s[c][pages, h].reshape(-1, D // 2)[:n], s[e][pages, h].reshape(-1, D // 32)[:n]
                else:
                    codes, exps = s[c][b, h, :n], s[e][b, h, :n]
                x = torch.empty((n, D), **f64)
                for half, shift in ((0, 0), (1, 4)):
                    w = (codes.long() >> shift) & 15
                    x[:, half::2] = steps[w & 7] * (1 - 2 * (w >> 3))
                kv.append(x * torch.exp2(exps.double() - 127.0).repeat_interleave(32, dim=-1))
            x = s["q"][b, :, h * G:(h + 1) * G].double().reshape(T * G, D) @ kv[0].t() / math.sqrt(D)
            seen = ctx + torch.arange(T, device="cuda").repeat_interleave(G)
            x.masked_fill_(torch.arange(n, device="cuda")[None] > seen[:, None], -math.inf)
            z = torch.logsumexp(x, dim=-1, keepdim=True)
            p = torch.exp(x - z)
            out[b, :, h * G:(h + 1) * G] = (p @ kv[1]).view(T, G, D)
            lse[b, h * G:(h + 1) * G] = z.view(T, G).t()
            mass[b, :n] += p.sum(dim=0)
    r = dict(out=out, lse=lse)
    return dict(r, mass=mass) if case["mass"] else r


def exact(case, seed):
    if case["kind"] == "pages":     # whole numbers: nothing to be off
        return None
    return {"rotary": _exact_rotary, "append": _exact_rotary, "handover": _exact_handover,
            "verify": _exact_verify}[case["kind"]](case, seed)
