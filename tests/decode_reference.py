"""Plain implementations of the decode step's operators in 64 bits, on the CPU, and how far
a right result may be from them.  They share nothing with the package."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U32 = 2.0 ** -24


def rounded_to(x, dtype):
    """Nearest value of a 16-bit type; of e4m3, bounded to 448."""
    if dtype == torch.float8_e4m3fn:
        return torch.where(x.isnan(), x, x.clamp(-448, 448)).float().to(dtype).double()
    return x.to(dtype).double()


def attend(q, k, v, table, lens, scale, n_blocks):
    """q [S, Hq, D]; k, v [block, P, H, D] (values, float64); table [S, B]; lens [S].
    Returns dict: out, lse, mass [S, B], and for the tolerance: `spread` = sum w |v|, `size` = the
    largest sum_i |q_i k_i| scale of a row, `top` = the largest |v|."""
    n, q_heads, dim = q.shape
    p, heads = k.shape[1], k.shape[2]
    g = q_heads // heads
    out, spread = torch.zeros(n, q_heads, dim, dtype=torch.float64), torch.zeros(n, q_heads, dim, dtype=torch.float64)
    lse, size = torch.full((n, q_heads), -math.inf, dtype=torch.float64), torch.zeros(n, q_heads, dtype=torch.float64)
    top = torch.zeros(n, q_heads, dtype=torch.float64)
    mass = torch.zeros(table.shape, dtype=torch.float64)
    for s in range(n):
        length = min(max(int(lens[s]), 0), table.shape[1] * p)
        cells = [(int(table[s, t // p]), t % p, t // p) for t in range(length) if 0 <= int(table[s, t // p]) < n_blocks]
        if not cells:
            continue
        page, row, entry = (torch.tensor(c) for c in zip(*cells))
        for h in range(q_heads):
            kk, vv, qq = k[page, row, h // g], v[page, row, h // g], q[s, h]
            a = (kk @ qq) * scale
            w = torch.softmax(a, 0)
            out[s, h], spread[s, h] = w @ vv, w @ vv.abs()
            lse[s, h] = torch.logsumexp(a, 0)
            size[s, h] = ((kk * qq).abs().sum(1) * abs(scale)).max()
            top[s, h] = vv.abs().max()
            mass[s].index_add_(0, entry, w)
    return dict(out=out, lse=lse, mass=mass, spread=spread, size=size, top=top)


def attend_bounds(ref, lens, dim, dtype):
    """|result - reference| of out, lse and mass.

    A score is a sum of dim products in 32 bits (exact products, dim additions), scaled: it is off by at
    most e = (dim + 4) 2^-24 size, plus 2^-24 of what it is compared with (below 2 size + 1) twice; a
    weight's relative error is twice that (both its numerator and the sum's), plus two roundings of exp2 and
    two of log2, 2^-22 each, plus the sums over the tokens: at most a rounding per step of 32 tokens and
    64 in the joins.  out: weights rounded to the 16-bit type (half a step, twice: numerator and sum), then the
    result itself; fp16 weights below the normal range are off by at most 2^-33 of the largest weight each."""
    u = HALF_STEP[dtype]
    steps = (lens.double().clamp(min=0) / 32 + 64)[:, None]
    e = (dim + 4) * U32 * ref["size"] + 4 * U32 * (ref["size"] + 1)
    rel = 2 * (e + 8 * 2.0 ** -22 + steps * U32)
    few = (lens.double().clamp(min=0) * 2.0 ** -33)[:, None] * ref["top"] if dtype == torch.float16 else 0 * ref["top"]
    out = (2 * u * (1 + 2 * u) + rel)[..., None] * ref["spread"] + few[..., None] + u * (1 + 2 * u) * ref["out"].abs() + 1e-30
    if dtype == torch.float16:
        out = out + 2.0 ** -24          # results below the normal range
    lse = rel + 4 * U32 * (ref["lse"].abs().nan_to_num(posinf=0) + 1) + 4 * U32 * ref["size"]
    weights = rel.max(1).values[:, None] * 2 + 4 * U32
    return out, lse, weights * (ref["mass"] + 1e-30) * (1 + 0 * ref["mass"])


def turned(x, positions, inv_freq, sections, rot, interleaved):
    """x [row, head, dim] in 64 bits; positions [axis, row]."""
    x = x.double().clone()
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    for i in range(rot // 2):
        a = positions[axis[i]].double() * inv_freq[i].double()
        c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
        i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        u, w = x[..., i1].clone(), x[..., i2].clone()
        x[..., i1], x[..., i2] = u * c - w * s, w * c + u * s
    return x


def evict(table, lens, mass, p, budget, first, last, cap):
    """One after the other: the lightest that may go, lower entries first."""
    table, mass = table.clone(), mass.clone()
    n, b = table.shape
    lens_out, count = lens.clone(), torch.zeros(n, dtype=torch.int32)
    ids, at = torch.full((n, cap), -1, dtype=torch.int32), torch.full((n, cap), -1, dtype=torch.int32)
    for s in range(n):
        length = min(max(int(lens[s]), 0), b * p)
        held = -(-length // p)
        may = [j for j in range(held) if first <= j < held - last]
        weight = lambda j: (math.inf, 1, j) if math.isnan(mass[s, j]) else (float(mass[s, j]), 0, j)  # noqa: E731
        go = sorted(sorted(may, key=weight)[:max(0, min(held - budget, len(may), cap))])
        gone = set(go)
        stay = [j for j in range(held) if j not in gone]
        row, m = table[s].clone(), mass[s].clone()
        table[s], mass[s] = -1, 0
        table[s, :len(stay)], mass[s, :len(stay)] = row[stay], m[stay]
        ids[s, :len(go)], at[s, :len(go)] = row[go], torch.tensor(go, dtype=torch.int32)
        lens_out[s], count[s] = length - p * len(go), len(go)
    return dict(table=table, lens=lens_out, mass=mass, ids=ids, at=at, count=count)
