"""Attention in 64 bits with bounds of what the 8-bit verify may be off by, and
inputs on which a lost or doubled token shows (no GPU needed).

The bounds follow the kernels' sums (u = 2^-24, half a step of fp32; the
exponential and its argument as in ``test_parity_q8``: |s| 2^-23 + 2^-20):

* A row's sum: 15 additions in a block of a lane, 2u for the compensated sum
  over all blocks whatever their number, four rescales of 5u (the factor's
  exponential 4u, the product u), 3 additions that join a row's lanes; then its
  records, ``steps`` of them one after the other in a set of lanes (at least two sets
  a row): a factor of 5u and an addition each, a rescale of 5u for every eighth;
  five joins of sets and waves, 6u each.  In all (15 + 2 + 20 + 3 + 5 + 30 = 75) u
  and 13/8 u a step: ``(80 + 2 steps) u`` of the sum.  No term grows with the
  number of tokens.
* A score: exact products, of which those that are not 0 round the sum: (terms + 4) u
  of the sum of their magnitudes.
* The log-sum-exp adds its logarithm's and its own roundings.
* O and the sum of the rounded probabilities: a matrix instruction takes in 32
  tokens and loses 2^-21 of what it adds up; a record has at most ``per + 2``
  of them, per being a workgroup's share in units of 32 tokens.  Then the records
  as above.
* P is rounded to bf16, off by 2^-8 of itself, in the numerator and in the
  denominator: 2^-8 (sum P|V| + |out|).  The result is rounded to bf16: 2^-8 |out|.

Inputs: ``aimed`` gives every query row a class of tokens (i mod C) that it looks
at evenly, every other token 2^-40 of them, and values that are the two digits
of a token's block number: a column of the result is the share of the class in
the blocks with that digit.  With B blocks a column, a lost block takes 1 / B of
it, more than the bound's 3 * 2^-8 while B is under 80.
"""
import torch

U = 2.0 ** -24
LN2 = 0.6931471805599453
AIM = 40.0      # log2 of what a row's class weighs beside any other token


def plan(ctx, T, G, Hkv, cus=256):
    """(units of a share, records of a row) at most, of the launch plan."""
    tiles = -(-G * T // 16)
    rg = -(-tiles // 10)
    rt = -(-tiles // rg)
    units = [-(-(c + T) // 32) for c in ctx]
    per = max(2, -(-sum(units) * Hkv * rg // cus))
    return per, (2 if rt <= 6 else 1) * (-(-max(units) // per) + 1)


def reference(q, K, V, ctx, scale, cus=256):
    """(out, lse, mass) of q [B][T][Hq][D] over float64 K, V [B][Hkv][n][D], and their bounds."""
    B, T, Hq, D = q.shape
    Hkv, n_cap = K.shape[1], K.shape[2]
    G = Hq // Hkv
    per, records = plan(ctx, T, G, Hkv, cus)
    sums = (80 + 2 * (records // 2 + 1)) * U
    weigh = sums + (per + 2) * 2.0 ** -21
    f = dict(dtype=torch.float64, device=q.device)
    out, lse, mass = torch.zeros((B, T, Hq, D), **f), torch.zeros((B, Hq, T), **f), torch.zeros((B, n_cap), **f)
    b_out, b_lse, b_mass = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(mass)
    for b, c in enumerate(ctx):
        n = c + T
        hidden = torch.arange(n, device=q.device)[None] > c + torch.arange(T, device=q.device).repeat_interleave(G)[:, None]
        for g in range(Hkv):
            hs = slice(g * G, (g + 1) * G)
            x = q[b, :, hs].double().reshape(T * G, D)
            s = (scale * x @ K[b, g, :n].t()).masked_fill(hidden, -torch.inf)
            terms = (x != 0).double() @ (K[b, g, :n] != 0).double().t()
            ds = scale * U * (terms + 4) * (x.abs() @ K[b, g, :n].abs().t())
            ds = (ds + s.abs() * 2.0 ** -23).masked_fill(hidden, 0.0).amax(dim=-1, keepdim=True) + 2.0 ** -20
            z = torch.logsumexp(s, dim=-1, keepdim=True)
            p = torch.exp(s - z)
            o, pv = p @ V[b, g, :n], p @ V[b, g, :n].abs()
            dp = 2 * (ds + sums)
            out[b, :, hs] = o.view(T, G, D)
            b_out[b, :, hs] = (2.0 ** -8 * (2 * o.abs() + pv) + (dp + 2 * weigh) * pv).view(T, G, D)
            lse[b, hs] = z.view(T, G).t()
            b_lse[b, hs] = (ds + sums + (z.abs() + 64) * 2.0 ** -22).view(T, G).t()
            mass[b, :n] += p.sum(dim=0)
            b_mass[b, :n] += (dp * p).sum(dim=0)
    return (out, lse, mass), (b_out, b_lse, b_mass + 2.0 ** -126 * Hq * T)


def beyond(got, want, bound):
    """Whether a result is off by more than its bound anywhere."""
    return bool((~((got.double() - want).abs() <= bound)).any())


def aimed(B, T, Hq, Hkv, D, rows, device="cpu"):
    """q (bf16), k_codes, k_exps, v_codes, v_exps, with ``rows`` (a multiple of 32) cache rows, and the scale.  The same
    value is held as two codes with their exponents, so that a row with another's exponent shows."""
    G = Hq // Hkv
    classes = min(64, D, T * G)
    i = torch.arange(rows, device=device)
    half, block = D // 2, i // 64

    def rows_of(cols, log2):       # value 2^log2 in the given columns
        odd = i % 3 == 1
        codes = torch.zeros((rows, D), dtype=torch.uint8, device=device)
        code = torch.where(odd, 0x40, 0x30).to(torch.uint8)           # 2 or 1/2
        for c in cols:
            codes[i, c] = code
        exps = torch.where(odd, 126 + log2, 128 + log2).to(torch.uint8)
        return (codes.expand(B, Hkv, rows, D).contiguous(), exps.expand(B, Hkv, rows).contiguous())
    k = rows_of([i % classes], 3)
    v = rows_of([block % half, half + block // half % half], 0)
    r = torch.arange(T * G, device=device)
    q = torch.zeros((B, T, Hq, D), dtype=torch.bfloat16, device=device)
    for g in range(Hkv):
        x = torch.zeros((T * G, D), dtype=torch.bfloat16, device=device)
        x[r, r % classes] = AIM / 8
        q[:, :, g * G:(g + 1) * G] = x.view(T, G, D)
    return q, (*k, *v), LN2


def values(codes, exps):
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(exps.double() - 127.0)[..., None]
