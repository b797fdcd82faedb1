"""The operators of the 8-bit key-value cache: their calls, and what those calls compute.

Four kinds of case:

* ``append``    rotary embedding of the new rows and the append of their keys
                and values, quantised, to the cache.
* ``quantise``  the rows of a 16- or 32-bit cache that a prefill left, into an
                8-bit one (a stack of layers in one call).
* ``verify``    attention of T new rows over the 8-bit cache with every token's
                attention mass; T = 1 without mass is a decode step.
* ``gather``    the draft's compact cache from the kept rows of every layer, as
                8-bit rows or read back as bf16.

A cache row of D values is D e4m3 codes and one exponent byte e, and stands for
``code * 2**(e - 127)``; e is the smallest number in [1, 254] that keeps the
row's largest finite magnitude within 448.  Codes are ``torch.float8_e4m3fn``,
exponents ``torch.uint8``.  A padded cache is [B][Hkv][n_cap][D] with exponents
[B][Hkv][n_cap]; a paged one [n_pages][Hkv][page][D] with [n_pages][Hkv][page].

Shapes are those of ``workloads`` (LLaVA-OV 7B and 72B, Qwen2.5-VL-32B, the
131K-token video and the small D = 64 configuration); ``draw`` spreads over the
ranges around them.
"""
import math
import random

import torch

own = False

E4M3, BF16, F32 = "e4m3", "bf16", "f32"
_BASE = 1.0e6


# ------------------------------------------------------------------ cases --
def _named(name, case):
    return dict(case, name=name) if name else case


def _append(name, B, T, hq, hkv, D, ctx_lo, ctx_hi, page=0, mrope=False):
    return _named(name, dict(kind="append", B=B, T=T, hq=hq, hkv=hkv, D=D, ctx_lo=ctx_lo,
                             ctx_hi=ctx_hi, page=page, mrope=mrope))


def _quantise(name, dtype, layers, B, hkv, D, len_lo, len_hi, page=0):
    return _named(name, dict(kind="quantise", dtype=dtype, layers=layers, B=B, hkv=hkv, D=D,
                             len_lo=len_lo, len_hi=len_hi, page=page))


def _verify(name, B, T, hq, hkv, D, ctx_lo, ctx_hi, page=0, mass=True):
    return _named(name, dict(kind="verify", B=B, T=T, hq=hq, hkv=hkv, D=D, ctx_lo=ctx_lo,
                             ctx_hi=ctx_hi, page=page, mass=mass))


def _gather(name, to, layers, B, hkv, D, m_lo, m_hi, n, keep_num, keep_den, page=0):
    return _named(name, dict(kind="gather", to=to, layers=layers, B=B, hkv=hkv, D=D, m_lo=m_lo,
                             m_hi=m_hi, n=n, keep_num=keep_num, keep_den=keep_den, page=page))


def listed():
    return [
        # The 7B target's six verify rows into a paged cache: a small call, all latency.
        _append("append-7b", 1, 6, 28, 4, 128, 6432, 6432, page=32),
        # The 72B target's whole prompt (64 frames and the text), one layer of its prefill.
        _append("append-72b-prompt", 1, 12800, 64, 8, 128, 0, 0),
        # One layer of the 7B draft's compact cache, made in bf16.
        _quantise("quantise-draft-7b", BF16, 1, 1, 4, 128, 787, 787),
        # The 7B target's cache of all 28 layers after its prefill.
        _quantise("quantise-7b", BF16, 28, 1, 4, 128, 6432, 6432),
        # The small configuration, D = 64: the smallest verify call.
        _verify("verify-tiny", 1, 5, 4, 1, 64, 1024, 1024),
        # The 7B draft's decode step over its compact cache: one row, no mass.
        _verify("verify-draft-7b", 1, 1, 28, 4, 128, 787, 787, mass=False),
        # One token of each of sixteen 7B sequences, ragged, paged: batched decoding.
        _verify("decode-batch-paged", 16, 1, 28, 4, 128, 2048, 16384, page=64, mass=False),
        # The headline: a layer of the 72B target's verify forward, 64 frames, gamma = 8.
        _verify("verify-72b", 1, 9, 64, 8, 128, 12800, 12800),
        # A ragged batch over a paged cache, one Qwen-32B layer.
        _verify("verify-32b-paged", 4, 9, 40, 8, 128, 16384, 33280, page=32),
        # One layer over a 131K-token video, gamma = 16: the longest context.
        _verify("verify-long", 1, 17, 64, 8, 128, 132096, 132096),
        # The 7B hand-over to a draft that keeps 8-bit rows: a tenth of the visual rows and the text.
        _gather("gather-7b", E4M3, 28, 1, 4, 128, 6272, 6272, 160, 1, 10),
        # The 72B hand-over, all 80 layers, to a draft whose cache is bf16.
        _gather("gather-72b-bf16", BF16, 80, 1, 8, 128, 12544, 12544, 256, 1, 10),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "quantise", "verify", "verify", "verify", "verify", "gather"])
    hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 4, 5, 7, 8])
    D = rng.choice([64, 128, 128])
    page = rng.choice([0, 0, 32, 64, 256])
    B = rng.choice([1, 1, 2, 3, 4])
    if kind == "append":
        T = rng.choice([rng.randint(1, 32), _log(rng, 1, 12800 // B)])
        ctx = _log(rng, 1, 30000)
        return _append(None, B, T, group * hkv, hkv, D, rng.randint(0, ctx), ctx, page=page,
                       mrope=rng.random() < 0.3)
    if kind == "verify":
        T = rng.choice([1, 1, rng.randint(2, 9), rng.randint(2, 17), rng.randint(2, 32)])
        B = rng.choice([B, rng.randint(1, 16)]) if T == 1 else B
        # at most the work of the longest listed one
        hi = _log(rng, 1, 132096 * min(1, 17 * 64 * 128 / (T * group * hkv * D)) / B)
        return _verify(None, B, T, group * hkv, hkv, D, rng.randint(hi // 3, hi), hi, page=page,
                       mass=T > 1 or rng.random() < 0.3)
    layers = rng.choice([1, 28, 64, 80])
    if kind == "quantise":
        dtype, hi = rng.choice([BF16, BF16, F32]), _log(rng, 1, 40000 // B)
        c = _quantise(None, dtype, 1, B, hkv, D, rng.randint(0, hi), hi, page=page)
        most = 550e6
    else:
        to, hi = rng.choice([E4M3, BF16, BF16, F32]), _log(rng, 20, 60000 // B)
        c = _gather(None, to, 1, B, hkv, D, rng.randint(hi // 2, hi), hi, rng.randint(1, 1024),
                    rng.randint(1, 50), 100, page=page)
        # at most 2 GB of cache behind it
        most = min(700e6, 2e9 * work(c)["bytes"] / (2 * B * (hi + c["n"]) * hkv * (D + 1)))
    return dict(c, layers=max(1, min(layers, int(most / work(c)["bytes"]))))


# ----------------------------------------------------------------- inputs --
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def _lengths(lo, hi, B):
    """Lengths of a ragged batch: the longest is hi, the others between."""
    r = random.Random(7919 * lo + 31 * hi + B)
    return [hi] + [r.randint(lo, hi) for _ in range(B - 1)]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cap(rows):
    """Row capacity of a padded 8-bit cache: a multiple of 32."""
    return max(32, -(-rows // 32) * 32)


def _power(e):
    """2**(e - 127) for whole numbers e in [1, 254]."""
    return torch.bitwise_left_shift(e.int(), 23).view(torch.float32)


def _to_8bit(x):
    """Codes and exponents of the rows of x (in its last dimension)."""
    x = x.float()
    top = torch.nan_to_num(x.abs(), nan=0.0, posinf=0.0).amax(dim=-1).view(torch.int32)
    # top = 2**(b - 127) * 1.m for its exponent b and mantissa m; 448 = 2**8 * 1.75
    e = ((top >> 23) - 8 + ((top & 0x7fffff) > 0x600000)).clamp(1, 254)
    return (x * _power(254 - e)[..., None]).to(torch.float8_e4m3fn), e.to(torch.uint8)


def _rows(g, shape):
    """Keys or values of one layer as a model has them: channels of different
    size, a few rows much larger or smaller than the rest."""
    x = torch.randn(shape, device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn(shape[-1:], device="cuda", generator=g))
    size = torch.exp(0.4 * torch.randn(shape[:-1] + (1,), device="cuda", generator=g))
    return x * size


def _cache(g, case, lens, layers=None):
    """An 8-bit cache of rows 0 .. lens[b] - 1; rows past them hold arbitrary codes."""
    B, hkv, D, P = (case[k] for k in ("B", "hkv", "D", "page"))
    table = None
    if P:
        need = [-(-n // P) for n in lens]
        n_pages = sum(need) + 3
        perm = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
        table = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
        o = 0
        for b in range(B):
            table[b, :need[b]] = perm[o:o + need[b]]
            o += need[b]
        shape = (n_pages, hkv, P, D)
    else:
        shape = (B, hkv, _cap(max(lens)), D)
    out = []
    for _ in range(2):
        parts = [_to_8bit(_rows(g, shape)) for _ in range(layers or 1)]
        out += [torch.stack([p[0].view(torch.uint8) for p in parts]).view(torch.float8_e4m3fn),
                torch.stack([p[1] for p in parts])] if layers else list(parts[0])
    return dict(kc=out[0], ke=out[1], vc=out[2], ve=out[3], table=table)


def _prepare_append(case, seed):
    g = _gen(seed)
    B, T, hq, hkv, D = (case[k] for k in ("B", "T", "hq", "hkv", "D"))
    lens = _lengths(case["ctx_lo"], case["ctx_hi"], B)
    ctx = _i32(lens)
    s = _cache(g, case, [n + T for n in lens])
    pos = ctx[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")[None]
    if case["mrope"]:
        lag = torch.randint(0, 64, (2, B, T), device="cuda", generator=g, dtype=torch.int32)
        pos = torch.cat([pos[None], torch.relu(pos[None] - lag)]).contiguous()
        s["sections"] = (D // 8, D // 4 - D // 16, D // 4 - D // 16)
    else:
        s["sections"] = None
    return dict(s, ctx=ctx, pos=pos.contiguous(), q=_rows(g, (B, T, hq, D)).bfloat16(),
                k_new=_rows(g, (B, T, hkv, D)).bfloat16(), v_new=_rows(g, (B, T, hkv, D)).bfloat16())


def _prepare_quantise(case, seed):
    g = _gen(seed)
    L, B, hkv, D = (case[k] for k in ("layers", "B", "hkv", "D"))
    lens = _lengths(case["len_lo"], case["len_hi"], B)
    dt = torch.bfloat16 if case["dtype"] == BF16 else torch.float32
    s = _cache(g, case, lens, L)
    cap = max(lens) + 5     # the prefill's own capacity
    src = [torch.stack([_rows(g, (B, hkv, cap, D)).to(dt) for _ in range(L)]) for _ in range(2)]
    return dict(s, k=src[0], v=src[1], lens=_i32(lens))


def _prepare_verify(case, seed):
    g = _gen(seed)
    B, T, hq, hkv, D = (case[k] for k in ("B", "T", "hq", "hkv", "D"))
    lens = _lengths(case["ctx_lo"], case["ctx_hi"], B)
    s = _cache(g, case, [n + T for n in lens])
    # queries whose scores are as wide as a model's, and, as a model's do, look
    # much at the first rows and at one row in fifty
    q = torch.randn((B, T, hq, D), device="cuda", generator=g)
    mean_q = q.view(B, T, hkv, hq // hkv, D).mean(dim=(1, 3))
    mean_q = 3.0 * mean_q / mean_q.norm(dim=-1, keepdim=True)
    for b, n in enumerate(lens):
        at = torch.randint(0, n + T, (max(1, (n + T) // 50),), device="cuda", generator=g)
        at = torch.cat([at, torch.zeros(1, dtype=at.dtype, device="cuda")]).unique()
        rows = torch.randn((at.numel(), hkv, D), device="cuda", generator=g) + mean_q[b][None]
        codes, exps = _to_8bit(rows)
        if case["page"]:
            pg, r = s["table"][b, at // case["page"]].long(), at % case["page"]
            s["kc"].view(torch.uint8)[pg, :, r] = codes.view(torch.uint8)
            s["ke"][pg, :, r] = exps
        else:
            s["kc"].view(torch.uint8)[b][:, at] = codes.view(torch.uint8).transpose(0, 1)
            s["ke"][b][:, at] = exps.transpose(0, 1)
    return dict(s, q=q.bfloat16(), ctx=_i32(lens), max_ctx=max(lens), mass=case["mass"])


def _prepare_gather(case, seed):
    g = _gen(seed)
    B, n = case["B"], case["n"]
    m = _lengths(case["m_lo"], case["m_hi"], B)
    keep = [x * case["keep_num"] // case["keep_den"] for x in m]
    k_cap = max(1, max(keep))
    idx = torch.full((B, k_cap), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        at = torch.randperm(m[b], device="cuda", generator=g)[:keep[b]].sort().values
        idx[b, :keep[b]] = at.to(torch.int32)
    s = _cache(g, case, [x + n for x in m], case["layers"])
    return dict(s, idx=idx, k=_i32(keep), m=_i32(m), tail=_i32([n] * B), to=case["to"],
                dst_cap=_cap(max(keep) + n), keep=keep, n=n)


def prepare(case, seed):
    s = {"append": _prepare_append, "quantise": _prepare_quantise, "verify": _prepare_verify,
         "gather": _prepare_gather}[case["kind"]](case, seed)
    return dict(s, kind=case["kind"])


# ------------------------------------------------------- the plain forms --
def _at(s, b, rows):
    """Where rows (same shape as b) of sequences b lie in a cache: the indices before and after the head's."""
    if s["table"] is None:
        return b, rows
    P = s["kc"].shape[-2]
    return s["table"][b, rows // P].long(), rows % P


def _plain_append(s):
    q, k, ctx = s["q"], s["k_new"], s["ctx"].long()
    B, T, _, D = q.shape
    h = D // 2
    theta = _BASE ** (-2.0 * torch.arange(h, dtype=torch.float64, device="cuda") / D)
    if s["sections"] is None:
        p = s["pos"].double()[..., None].expand(B, T, h)
    else:
        i = torch.arange(h, device="cuda")
        axis = (i >= s["sections"][0]).long() + (i >= s["sections"][0] + s["sections"][1]).long()
        p = s["pos"].double()[axis].permute(1, 2, 0)
    ang = (p * theta)[:, :, None, :]
    cos, sin = torch.cos(ang), torch.sin(ang)

    def rotate(x):
        x1, x2 = x.double().chunk(2, dim=-1)
        return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1).float().bfloat16()

    t = torch.arange(T, device="cuda")
    at, row = _at(s, torch.arange(B, device="cuda")[:, None].expand(B, T), ctx[:, None] + t)
    kc, ke = _to_8bit(rotate(k))
    vc, ve = _to_8bit(s["v_new"])
    s["kc"].view(torch.uint8)[at, :, row] = kc.view(torch.uint8)
    s["vc"].view(torch.uint8)[at, :, row] = vc.view(torch.uint8)
    s["ke"][at, :, row] = ke
    s["ve"][at, :, row] = ve
    return dict(q=rotate(q), k_codes=s["kc"], k_exps=s["ke"], v_codes=s["vc"], v_exps=s["ve"])


def _plain_quantise(s):
    L, B, hkv, cap, _ = s["k"].shape
    b, i = torch.nonzero(torch.arange(cap, device="cuda")[None] < s["lens"][:, None], as_tuple=True)
    at, row = _at(s, b, i)
    for x, c, e in (("k", "kc", "ke"), ("v", "vc", "ve")):
        codes, exps = _to_8bit(s[x][:, b, :, i])
        s[c].view(torch.uint8)[:, at, :, row] = codes.view(torch.uint8)
        s[e][:, at, :, row] = exps
    return dict(k_codes=s["kc"], k_exps=s["ke"], v_codes=s["vc"], v_exps=s["ve"])


def _values(codes, exps, table):
    """The fp32 values of a cache's rows as [B][Hkv][rows][D]."""
    if table is not None:
        at = table.clamp_min(0).long()
        codes = codes.view(torch.uint8)[at].transpose(1, 2).flatten(2, 3).view(torch.float8_e4m3fn)
        exps = exps[at].transpose(1, 2).flatten(2, 3)
    return codes.float() * _power(exps)[..., None]


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


def _plain_gather(s):
    L, hkv, D = s["kc"].shape[0], s["kc"].shape[2], s["kc"].shape[-1]
    B, cap = s["idx"].shape[0], s["dst_cap"]
    r = torch.arange(cap, device="cuda")[None]
    kept = r < s["k"][:, None]
    b, i = torch.nonzero(r < (s["k"] + s["tail"])[:, None], as_tuple=True)
    first = s["idx"].long().gather(1, r.clamp_max(s["idx"].shape[1] - 1).expand(B, cap))
    src = torch.where(kept, first, s["m"].long()[:, None] + r - s["k"].long()[:, None])
    at, row = _at(s, b, src[b, i])
    out = {}
    for name, c, e in (("k", "kc", "ke"), ("v", "vc", "ve")):
        codes, exps = s[c].view(torch.uint8)[:, at, :, row], s[e][:, at, :, row]
        if s["to"] == E4M3:
            d = torch.zeros((L, B, hkv, cap, D), dtype=torch.uint8, device="cuda")
            x = torch.zeros((L, B, hkv, cap), dtype=torch.uint8, device="cuda")
            d[:, b, :, i], x[:, b, :, i] = codes, exps
            out[name + "_codes"], out[name + "_exps"] = d.view(torch.float8_e4m3fn), x
        else:
            dt = torch.bfloat16 if s["to"] == BF16 else torch.float32
            d = torch.zeros((L, B, hkv, cap, D), dtype=dt, device="cuda")
            x = codes.view(torch.float8_e4m3fn).float() * _power(exps)[..., None]
            d[:, b, :, i] = x.to(dt)
            out[name] = d
    return out


# --------------------------------------------------- the framework's calls --
def _own_run(s):
    import paper_2603_19610_amd as pv
    cache = (s["kc"], s["ke"], s["vc"], s["ve"])
    table = s["table"]
    if s["kind"] == "append":
        rows = (s["q"], s["k_new"], s["v_new"], s["pos"], s["ctx"])
        if table is None:
            q = pv.rope_append_q8(*rows, *cache, base=_BASE, sections=s["sections"])
        else:
            q = pv.rope_append_q8_paged(*rows, *cache, table, base=_BASE, sections=s["sections"])
        return dict(q=q, k_codes=s["kc"], k_exps=s["ke"], v_codes=s["vc"], v_exps=s["ve"])
    if s["kind"] == "quantise":
        if table is None:
            pv.quantize_kv(s["k"], s["v"], s["lens"], *cache)
        else:
            pv.quantize_kv_paged(s["k"], s["v"], s["lens"], *cache, table)
        return dict(k_codes=s["kc"], k_exps=s["ke"], v_codes=s["vc"], v_exps=s["ve"])
    if s["kind"] == "verify":
        kw = dict(max_ctx=s["max_ctx"], want_mass=s["mass"])
        if table is None:
            out, mass, lse = pv.verify_attn_q8(s["q"], *cache, s["ctx"], **kw)
        else:
            out, mass, lse = pv.verify_attn_q8_paged(s["q"], *cache, table, s["ctx"], **kw)
        return dict(out=out, lse=lse, mass=mass) if s["mass"] else dict(out=out, lse=lse)
    dt = {E4M3: torch.float8_e4m3fn, BF16: torch.bfloat16, F32: torch.float32}[s["to"]]
    sel = (s["idx"], s["k"], s["m"], s["tail"], s["dst_cap"])
    if table is None:
        got = pv.gather_kv_q8(*cache, *sel, dtype=dt)
    else:
        got = pv.gather_kv_q8_paged(*cache, table, *sel, dtype=dt)
    return dict(zip(("k_codes", "k_exps", "v_codes", "v_exps") if s["to"] == E4M3 else ("k", "v"), got))


def run(s):
    if own:
        return _own_run(s)
    return {"append": _plain_append, "quantise": _plain_quantise, "verify": _plain_verify,
            "gather": _plain_gather}[s["kind"]](s)


# ------------------------------------------------------- work and accuracy --
def work(case):
    kind, B, hkv, D = case["kind"], case["B"], case["hkv"], case["D"]
    if kind == "append":
        n, hq = B * case["T"], case["hq"]
        size = n * (2 * (2 * hq + 2 * hkv) * D + 2 * hkv * (D + 1) + (12 if case["mrope"] else 4)) + 4 * B
        return dict(bytes=size, flops=n * (3 * (hq + hkv) + 2 * 2 * hkv) * D)
    if kind == "quantise":
        rows = case["layers"] * hkv * sum(_lengths(case["len_lo"], case["len_hi"], B))
        e = 2 if case["dtype"] == BF16 else 4
        return dict(bytes=2 * rows * (D * e + D + 1) + 4 * B, flops=2 * rows * 2 * D)
    if kind == "verify":
        T, hq = case["T"], case["hq"]
        rows = sum(n + T for n in _lengths(case["ctx_lo"], case["ctx_hi"], B))
        size = 2 * rows * hkv * (D + 1) + 2 * B * T * hq * D * 2 + 4 * B * hq * T + 4 * B
        return dict(bytes=size + (4 * rows if case["mass"] else 0), flops=4 * rows * hq * T * D)
    m = _lengths(case["m_lo"], case["m_hi"], B)
    kept = sum(x * case["keep_num"] // case["keep_den"] for x in m)
    row = {E4M3: D + 1, BF16: 2 * D, F32: 4 * D}[case["to"]]
    moved = case["layers"] * hkv * (kept + B * case["n"])
    return dict(bytes=2 * moved * (D + 1 + row) + 4 * kept, flops=2 * moved * D)


def _scaled(x):
    """The rows of x as multiples of their scale, unrounded, in 64 bits."""
    x = x.double()
    top = x.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp_min(2.0 ** -140) / 448.0)).clamp(-126, 127)
    e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, e)
    e = torch.where(448.0 * torch.exp2(e) < top, e + 1, e).clamp(-126, 127)
    return x * torch.exp2(-e)


def _exact_append(case, seed):
    s = _prepare_append(case, seed)
    B, T, P = case["B"], case["T"], case["page"]
    h = case["D"] // 2
    cuts = (h, h, h) if s["sections"] is None else (s["sections"][0], s["sections"][0] + s["sections"][1], h)
    pos = s["pos"].double() if s["sections"] is not None else s["pos"].double()[None]
    turn = torch.empty((B, T, 1, h), dtype=torch.complex128, device="cuda")
    for i in range(h):
        axis = 0 if i < cuts[0] else 1 if i < cuts[1] else 2
        a = pos[axis if pos.shape[0] == 3 else 0] * math.pow(_BASE, -i / h)
        turn[:, :, 0, i] = torch.polar(torch.ones_like(a), a)

    def rot(x):
        z = torch.complex(x[..., :h].double(), x[..., h:].double()) * turn
        return torch.cat([z.real, z.imag], dim=-1)

    q = rot(s["q"])
    # an appended row is that of a bf16 cache, in 8 bits
    k, v = _scaled(rot(s["k_new"]).to(torch.bfloat16)), _scaled(s["v_new"])
    kc, vc = s["kc"].double(), s["vc"].double()
    lens = s["ctx"].tolist()
    for b in range(B):
        i = torch.arange(lens[b], lens[b] + T, device="cuda")
        for c, x in ((kc, k), (vc, v)):
            if P:
                c[s["table"][b, i // P].long(), :, i % P] = x[b]
            else:
                c[b, :, lens[b]:lens[b] + T] = x[b].transpose(0, 1)
    return dict(q=q, k_codes=kc, k_exps=None, v_codes=vc, v_exps=None)


def _exact_quantise(case, seed):
    s = _prepare_quantise(case, seed)
    P, out = case["page"], {}
    for name, c, x in (("k_codes", "kc", "k"), ("v_codes", "vc", "v")):
        d = torch.empty(s[c].shape, dtype=torch.float64, device="cuda")
        for layer in range(case["layers"]):
            d[layer] = s[c][layer].double()
            for b, n in enumerate(s["lens"].tolist()):
                rows = _scaled(s[x][layer, b, :, :n])
                if P:
                    i = torch.arange(n, device="cuda")
                    d[layer][s["table"][b, i // P].long(), :, i % P] = rows.transpose(0, 1)
                else:
                    d[layer, b, :, :n] = rows
        out[name] = d
    return dict(out, k_exps=None, v_exps=None)


def _exact_verify(case, seed):
    s = _prepare_verify(case, seed)
    B, T, hq, hkv, D, P = (case[k] for k in ("B", "T", "hq", "hkv", "D", "page"))
    G = hq // hkv
    n_cap = s["table"].shape[1] * P if P else s["kc"].shape[2]
    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse = torch.zeros((B, T, hq, D), **f64), torch.zeros((B, hq, T), **f64)
    mass = torch.zeros((B, n_cap), **f64)
    for b, ctx in enumerate(s["ctx"].tolist()):
        n = ctx + T
        for h in range(hkv):
            kv = []
            for c, e in (("kc", "ke"), ("vc", "ve")):
                if P:
                    pages = s["table"][b, :-(-n // P)].long()
                    codes = s[c].view(torch.uint8)[pages, h].reshape(-1, D)[:n].view(torch.float8_e4m3fn)
                    exps = s[e][pages, h].reshape(-1)[:n]
                else:
                    codes, exps = s[c][b, h, :n], s[e][b, h, :n]
                kv.append(codes.double() * torch.exp2(exps.double() - 127.0)[:, None])
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


def _exact_gather(case, seed):
    s = _prepare_gather(case, seed)
    L, B, hkv, D, P = (case[k] for k in ("layers", "B", "hkv", "D", "page"))
    out = {}
    for name, c, e in (("k", "kc", "ke"), ("v", "vc", "ve")):
        d = torch.zeros((L, B, hkv, s["dst_cap"], D), dtype=torch.float64, device="cuda")
        for b in range(B):
            m = int(s["m"][b])
            rows = torch.cat([s["idx"][b, :s["keep"][b]].long(), torch.arange(m, m + s["n"], device="cuda")])
            for layer in range(L):
                if P:
                    pages = s["table"][b, rows // P].long()
                    codes, exps = s[c].view(torch.uint8)[layer, pages, :, rows % P], s[e][layer, pages, :, rows % P]
                else:
                    codes = s[c].view(torch.uint8)[layer, b, :, rows].transpose(0, 1)
                    exps = s[e][layer, b, :, rows].transpose(0, 1)
                x = codes.contiguous().view(torch.float8_e4m3fn).double()
                if s["to"] != E4M3:
                    x = x * torch.exp2(exps.double() - 127.0)[..., None]
                d[layer, b, :, :rows.numel()] = x.transpose(0, 1)
        out[name] = d
    if s["to"] == E4M3:
        return dict(k_codes=out["k"], k_exps=None, v_codes=out["v"], v_exps=None)
    return out


def exact(case, seed):
    return {"append": _exact_append, "quantise": _exact_quantise, "verify": _exact_verify,
            "gather": _exact_gather}[case["kind"]](case, seed)
