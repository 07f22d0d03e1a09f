"""Attention of many rows, a cache in 4 bits and normed heads in plain 64-bit arithmetic on the CPU, and how far a right
result may be from them.  Nothing here is shared with the package."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U32 = 2.0 ** -24
NUMBERS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
POWERS = {torch.bfloat16: (-126, 125), torch.float16: (-23, 13)}


def fp4_values(rows, heads, dim):
    """rows [..., heads * dim / 32 * 17] (uint8), the bytes of tokens: [..., heads, dim] in 64 bits."""
    n = heads * dim // 2
    code = torch.stack([rows[..., :n] & 15, rows[..., :n] >> 4], -1).flatten(-2).long()
    v = NUMBERS[code & 7] * torch.where(code >= 8, -1.0, 1.0).double()
    byte = rows[..., n:].double()
    power = torch.where(byte == 255, float("nan"), torch.exp2(byte - 127))
    return (v.unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2).unflatten(-1, (heads, dim))


def fp4_rows(x, dtype):
    """x [..., heads, dim] as bytes of tokens: each number the nearest of those there are, the even place of two as near."""
    lo, hi = POWERS[dtype]
    g = x.double().unflatten(-1, (-1, 32))
    largest = g.abs().amax(-1)
    odd = ~torch.isfinite(largest)
    e = torch.floor(torch.log2(torch.where(odd | (largest == 0), 2.0 ** -1000, largest))).clamp(min=-1000) - 2
    e = e.clamp(lo, hi)
    off = (g.abs().nan_to_num(0, 0)[..., None] / torch.exp2(e)[..., None, None] - NUMBERS).abs()
    code = off.argmin(-1)
    other = (code + 1).clamp(max=7)
    tie = (off.gather(-1, code[..., None]) == off.gather(-1, other[..., None]))[..., 0] & (other != code)
    code = torch.where(tie & (code % 2 == 1), other, code) + 8 * torch.signbit(g).long()
    code = torch.where(odd[..., None], 0, code).flatten(-3).to(torch.uint8)
    byte = torch.where(odd, 255, (e + 127).nan_to_num(0).long()).flatten(-2).to(torch.uint8)
    return torch.cat([code[..., 0::2] | code[..., 1::2] << 4, byte], -1)


def rows(q, k, v, table, lens, starts, scale, causal, n_blocks):
    """q [R, Hq, D]; k, v [block, P, H, D] (values, 64 bits).  Rows that belong to no request are NaN in what is returned:
    out, lse, and for the tolerance spread = sum w |v|, size, top and seen (tokens of each row)."""
    r, q_heads, dim = q.shape
    p, heads = k.shape[1], k.shape[2]
    group = q_heads // heads
    nan = float("nan")
    out, spread = (torch.full((r, q_heads, dim), nan, dtype=torch.float64) for _ in range(2))
    lse, size, top = (torch.full((r, q_heads), nan, dtype=torch.float64) for _ in range(3))
    tokens = torch.zeros(r, dtype=torch.float64)
    for s in range(len(lens)):
        a, b = int(starts[s]), min(int(starts[s + 1]), r)
        most = table.shape[1] * p
        length = min(max(int(lens[s]), 0), most)
        at = [t for t in range(length) if 0 <= int(table[s, t // p]) < n_blocks]
        for part in (out, spread, size, top):
            part[a:b] = 0
        lse[a:b] = -math.inf
        if not at or a >= b:
            continue
        place = torch.tensor(at)
        page, row = torch.tensor([int(table[s, t // p]) for t in at]), place % p
        m = int(starts[s + 1]) - a
        upto = int(lens[s]) - m + 1 + torch.arange(b - a) if causal else torch.full((b - a,), length)
        sees = place[None] < upto[:, None]
        tokens[a:b] = sees.sum(1).double()
        for h in range(q_heads):
            kk, vv, qq = k[page, row, h // group], v[page, row, h // group], q[a:b, h].double()
            x = (qq[:, None, :] * kk[None]).sum(-1) * scale if torch.isinf(kk).any() or torch.isnan(kk).any() else qq @ kk.t() * scale
            x = torch.where(sees, x, -math.inf)
            any_ = sees.any(1)
            w = torch.where(any_[:, None], torch.softmax(x, 1), 0.0)
            lse[a:b, h] = torch.logsumexp(x, 1)
            if torch.isfinite(vv).all():
                out[a:b, h] = w @ vv
            else:       # what is not seen makes no difference
                out[a:b, h] = torch.where(sees[..., None], w[..., None] * vv[None], 0.0).sum(1)
            fine = vv.nan_to_num(0, 0, 0).abs()
            spread[a:b, h] = w.nan_to_num(0) @ fine
            size[a:b, h] = torch.where(sees, qq.abs().nan_to_num(0) @ kk.abs().nan_to_num(0, 0).t() * abs(scale), 0.0).amax(1)
            top[a:b, h] = fine.max()
    return dict(out=out, lse=lse, spread=spread, size=size, top=top, tokens=tokens)


def rows_bounds(ref, dim, dtype, splits=512):
    """|result - reference| of out and lse.

    A score is a sum of dim products in 32 bits (exact products, dim additions), scaled: off by at most
    e = (dim + 4) 2^-24 size, and 2^-24 of what it is compared with (below 2 size + 1) twice; a weight's relative error is
    that, and 2^-22 of exp2 and log2 twice each.  Sums of weights add up half of the tokens one after the other, then
    two halves and the splits; sums of values take a step for 16 tokens.  So much for numerator and for sum.  out: weights are rounded
    to the 16-bit type, half a step each, then the result is; fp16 has weights of 2^12 and more for the largest and steps of
    2^-24, half of which are 2^-37 of it."""
    u = HALF_STEP[dtype]
    tokens = ref["tokens"][:, None]
    e = (dim + 4) * U32 * ref["size"] + 4 * U32 * (ref["size"] + 1)
    rel = 2 * (e + 8 * 2.0 ** -22) + (tokens / 2 + tokens / 16 + 4 * splits + 64) * U32
    few = tokens * 2.0 ** -37 * ref["top"] if dtype == torch.float16 else 0 * ref["top"]
    out = (u + rel)[..., None] * ref["spread"] * (1 + 2 * u) + few[..., None] + u * (1 + 2 * u) * ref["out"].abs() + 1e-30
    if dtype == torch.float16:
        out = out + 2.0 ** -24
    lse = rel + 4 * U32 * (ref["lse"].abs().nan_to_num(posinf=0) + 1) + 4 * U32 * ref["size"]
    return out, lse


def normed(x, weight, eps):
    x = x.double()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
