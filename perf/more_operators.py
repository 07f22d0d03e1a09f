"""Attention of many rows over the paged KV cache, and the cache in 4 bits, as cases that can be timed and compared.

  rows    several rows of every request (a prompt or a chunk of one, drafted tokens, a decoder's rows beside
          an encoder's states) over the pages it holds: up to each row's own place, or over all of them
  attend  one new token of every request over a cache held in 4 bits
  put     new tokens: q and k are normed head by head and get their rotary positions in the same pass, k and v
          go into their pages, in 16 bits or in 4

Where `own` is false, `run` computes them from elementary torch operations in 32 bits, rounded
once at the end; where it is true, through the package's decoder.

A row of a 4-bit cache is, token by token, n_kv_heads * dim / 2 bytes of pairs (the even dimension in the low
half) and n_kv_heads * dim / 32 bytes of exponents: 32 dimensions of a head share one, and a stored
number is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives times 2^(exponent byte - 127).
"""
import math

import numpy as np
import torch

own = False

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _rows(n_seqs, new, past, heads, group, dim, tokens, **opt):
    c = dict(op="rows", n_seqs=n_seqs, new=new, past=past, heads=heads, group=group, dim=dim, tokens=tokens, x="bf16", kv="16",
             causal=True, spread="equal", lse=False, holes=0.0, stale=False, behind=0, layers=1, block_first=False, shape_seed=1)
    c.update(opt)
    return c


def _attend(n_seqs, longest, heads, group, dim, tokens, **opt):
    c = dict(op="attend", n_seqs=n_seqs, longest=longest, heads=heads, group=group, dim=dim, tokens=tokens, x="bf16", kv="4",
             spread="lognormal", mass=False, lse=False, holes=0.0, stale=False, layers=1, block_first=False, shape_seed=1)
    c.update(opt)
    return c


def _put(n_seqs, new, past, heads, group, dim, tokens, **opt):
    c = dict(op="put", n_seqs=n_seqs, new=new, past=past, heads=heads, group=group, dim=dim, tokens=tokens, x="bf16", kv="16",
             norm=True, axes=1, rot=dim, interleaved=False, behind=0, layers=1, block_first=False, shape_seed=1)
    c.update(opt)
    return c


def listed():
    named = {
        # the smallest there is a configuration for: a few drafted tokens of two short requests, all latency
        "rows_tiny": _rows(2, 7, 90, 2, 2, 64, 16, layers=2),
        # four fresh prompts of a Llama-3-8B-shaped model: 8192 tokens in all
        "rows_prompts": _rows(4, 2048, 0, 8, 4, 128, 16),
        # a chunk of 1024 tokens of a 70B-shaped request that is 30000 tokens long already
        "rows_chunk_long_70b": _rows(1, 1024, 30000, 8, 8, 128, 32),
        # five drafted tokens of 16 requests that are to be verified, a cache in 8 bits
        "rows_drafts_fp8": _rows(16, 5, 8000, 8, 5, 128, 16, kv="8", spread="ragged", lse=True, block_first=True),
        # a decoder's rows over an encoder's states: every row sees all of them
        "rows_cross": _rows(24, 448, 1500, 12, 1, 64, 16, x="fp16", causal=False, spread="ragged", lse=True),
        # blocks of 5 tokens, 3 heads of 96 in 4 bits, pages that are not there, requests without rows, padding behind
        "rows_ragged_fp4": _rows(9, 300, 700, 3, 3, 96, 5, x="fp16", kv="4", spread="ragged", lse=True, holes=0.1, stale=True,
                                 behind=61, layers=2),
        # the smallest attention of one token over a 4-bit cache
        "attend_fp4_tiny": _attend(3, 100, 2, 2, 64, 16, layers=2, lse=True),
        # a large batch whose cache is held in 4 bits, weights kept for eviction
        "attend_fp4_batch": _attend(128, 4096, 8, 5, 128, 16, mass=True, block_first=True),
        # the 70B-shaped long context in 4 bits: 4 requests of 32768 tokens
        "attend_fp4_long_70b": _attend(4, 32768, 8, 8, 128, 32, spread="equal"),
        # a decode step of 64 requests of a model that norms its heads
        "put_norm_decode": _put(64, 1, 30000, 8, 4, 128, 16, layers=2),
        # prompts of 8192 tokens in all, normed heads, into 4 bits
        "put_norm_prompts_fp4": _put(4, 2048, 0, 8, 4, 128, 16, kv="4"),
        # half of each head rotates, neighbours paired, into 4 bits in blocks of 5, no norms, rows of padding behind
        "put_ragged_fp4": _put(7, 300, 900, 3, 4, 96, 5, x="fp16", kv="4", norm=False, rot=48, interleaved=True, behind=61),
    }
    return [dict(c, name=n) for n, c in named.items()]


def draw(rng):
    pick = rng.choice
    logu = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))  # noqa: E731
    op = pick(["rows", "rows", "rows", "attend", "attend", "put"])
    heads, group = pick([(8, 4), (8, 4), (8, 8), (8, 5), (1, 4), (1, 8), (2, 2), (4, 7), (3, 3), (2, 16), (1, 24), (12, 1)])
    kv = pick(["16", "16", "8", "4"]) if op == "rows" else pick(["16", "4"]) if op == "put" else "4"
    dim = pick([128, 128, 128, 64, 32, 96, 192, 256] if kv == "4" else [128, 128, 128, 64, 40, 80, 96, 192, 256])
    common = dict(shape_seed=rng.randrange(1 << 30), x=pick(["bf16", "bf16", "fp16"]), layers=pick([1, 2]),
                  block_first=pick([False, False, True]))
    tokens = pick([16, 16, 16, 32, 8, 5, 24])
    if op == "put":
        n_seqs = logu(1, 128)
        new = pick([1, 1, logu(2, max(3, min(8192, (32 << 20) // (heads * group * dim)) // n_seqs))])
        return _put(n_seqs, new, pick([0, logu(1, 4000), logu(4000, 120000)]), heads, group, dim, tokens, kv=kv,
                    norm=True if kv == "16" else pick([True, True, False]), axes=pick([1, 1, 3]), rot=pick([dim, dim, dim // 16 * 8]),
                    interleaved=pick([False, True]), behind=pick([0, 0, 13]), **common)
    common.update(spread=pick(["equal", "ragged"]), lse=pick([False, True]), holes=pick([0.0, 0.0, 0.05]), stale=pick([False, True]))
    row = 2 * heads * dim * 2 * common["layers"]
    if op == "attend":
        longest = logu(1, 131072)
        most = min((400 << 20) // row, (1 << 30) // (heads * group * dim))
        longest = min(longest, most)
        n_seqs = max(1, min(logu(1, 200), most // longest))
        common["spread"] = pick(["lognormal", common["spread"]])
        return _attend(n_seqs, longest, heads, group, dim, tokens, mass=pick([False, True]), **common)
    new = pick([logu(1, 12), logu(1, 2048)])
    n_seqs = logu(1, 64)
    causal = pick([True, True, False])
    past = pick([0 if causal else logu(1, 100), logu(1, 4000), logu(1000, 60000)])
    # no more products than 600 of the largest heads' GFLOP, and no more scores or rows than fit easily
    while n_seqs * (new + past) * row > 400 << 20 or n_seqs * new * heads * group * (new + past) * max(dim, 128) > 150 << 30 \
            or n_seqs * new * heads * group * dim > 64 << 20:
        if n_seqs > 1:
            n_seqs = (n_seqs + 1) // 2
        elif past > new:
            past //= 2
        else:
            new = (new + 1) // 2
    return _rows(n_seqs, new, past, heads, group, dim, tokens, kv=kv, causal=causal, behind=pick([0, 0, 13]),
                 **common)


# ---- what a case says of its requests (the same for every seed) -----------------------------------

def _lengths(case, longest):
    """How long each request is: all as long as the longest, lognormal around an eighth of
    it, or anything from nothing on."""
    rng, n = np.random.default_rng(case["shape_seed"]), case["n_seqs"]
    if case["spread"] == "equal":
        lens = np.full(n, longest)
    elif case["spread"] == "ragged":
        lens = rng.integers(0, longest + 1, n)
        lens[1::4] = rng.integers(0, 2, lens[1::4].size)
    else:
        lens = np.clip(np.rint(rng.lognormal(math.log(max(1.0, longest / 8)), 0.8, n)), max(1, longest // 128), longest)
    lens[0] = longest
    return lens.astype(np.int64)


def _counts(case):
    """(new rows, tokens attended over) of each request.  Rows that see up to their own place are the request's last tokens."""
    new = _lengths(case, case["new"])
    if case["spread"] == "equal":
        past = np.full(case["n_seqs"], case["past"])
    else:
        past = np.random.default_rng(case["shape_seed"] + 3).integers(0, case["past"] + 1, case["n_seqs"])
        past[0] = case["past"]
    return new, past + new if case["causal"] else past


def _blocks(lens, tokens):
    return -(-lens // tokens)


def _present(case, lens):
    """Which entries of the requests' tables name a page: [request, entry]."""
    held = _blocks(lens, case["tokens"])
    at = np.arange(max(1, int(held.max())))[None] < held[:, None]
    if case.get("holes"):
        at &= np.random.default_rng(case["shape_seed"] + 1).random(at.shape) >= case["holes"]
    return at


def _in_blocks(case, lens):
    """Tokens of each entry that is a page: [request, entry]."""
    at, p = _present(case, lens), case["tokens"]
    return np.clip(lens[:, None] - np.arange(at.shape[1])[None] * p, 0, p) * at


def _put_counts(case):
    few, n = np.random.default_rng(case["shape_seed"]), case["n_seqs"]
    new = np.full(n, case["new"]) if case["new"] == 1 else few.integers((case["new"] + 1) // 2, case["new"] + 1, n)
    return new, few.integers(case["past"] // 2, case["past"] + 1, n)


def _sections(case):
    """Pairs of each axis: time, height, width in about 1 : 1.5 : 1.5."""
    pairs = case["rot"] // 2
    if case["axes"] == 1:
        return (pairs,)
    t = pairs // 4
    h = (pairs - t) // 2
    return (t, h, pairs - t - h)


def _type(case):
    return torch.float16 if case["x"] == "fp16" else torch.bfloat16


def _scales(case):
    return (0.03, 0.0125) if case["kv"] == "8" else (1.0, 1.0)


def _token_bytes(case):
    """Bytes of one token's K or V."""
    n = case["heads"] * case["dim"]
    return {"16": 2 * n, "8": n, "4": n * 17 // 32}[case["kv"]]


# ---- a cache in 4 bits ----------------------------------------------------------------------------

def _split_fp4(case, x):
    """x [..., head, dim] in 32 bits: what 32 dimensions are multiples of, [..., head, dim / 32], as the power of 2's exponent, and
    the nearest of VALUES to each multiple (ties to the even place among them) with its sign."""
    g = x.unflatten(-1, (-1, 32))
    low, high = (-23, 13) if case["x"] == "fp16" else (-126, 125)
    exponent = (torch.frexp(g.abs().amax(-1))[1] - 3).clamp(low, high)
    exponent = torch.where(g.abs().amax(-1) > 0, exponent, torch.full_like(exponent, low))
    m = torch.ldexp(g.abs(), -exponent[..., None])
    code = sum((m >= t if odd else m > t).to(torch.uint8)
               for t, odd in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)))
    return exponent, (code + 8 * torch.signbit(g).to(torch.uint8)).flatten(-2)


def _to_fp4(case, x):
    """x [..., head, dim] as the bytes of a token: [..., n]."""
    exponent, code = _split_fp4(case, x)
    code = code.flatten(-2)
    return torch.cat([code[..., 0::2] | code[..., 1::2] << 4, (exponent + 127).to(torch.uint8).flatten(-2)], -1)


def _from_fp4(case, t):
    """The bytes of a token, [..., n], as what they stand for: [..., head, dim] in 32 bits."""
    n = case["heads"] * case["dim"] // 2
    code = torch.stack([t[..., :n] & 15, t[..., :n] >> 4], -1).flatten(-2).int()
    value = torch.tensor(VALUES + tuple(-v for v in VALUES), device=t.device)[code]
    value = torch.ldexp(value.unflatten(-1, (-1, 32)), (t[..., n:].int() - 127)[..., None])
    return value.flatten(-2).unflatten(-1, (case["heads"], case["dim"]))


# ---- inputs ---------------------------------------------------------------------------------------

def _table(rng, present, n_blocks):
    table = np.full(present.shape, -1, np.int32)
    table[present] = rng.permutation(n_blocks)[:int(present.sum())]
    return torch.from_numpy(table).cuda()


def _planes(s, which):
    """K (0) or V (1) of the case's layer: [block, token, ...], in the cache's own bytes."""
    c, cache = s["case"], s["cache"]
    at = c["layers"] - 1
    return cache[:, at, which] if c["block_first"] else cache[at, which]


def _new_values(case, n_blocks, g):
    """N(0, 1) in the 16-bit type, laid out as the cache."""
    inner = (case["tokens"], case["heads"], case["dim"])
    dims = (n_blocks, case["layers"], 2) + inner if case["block_first"] else (case["layers"], 2, n_blocks) + inner
    return torch.empty(dims, dtype=_type(case), device="cuda").normal_(generator=g)


def _to_cache_type(case, v):
    """Values of the 16-bit type as the cache holds them."""
    if case["kv"] == "16":
        return v
    if case["kv"] == "4":
        return _to_fp4(case, v.float())
    out = torch.empty(v.shape, dtype=torch.uint8, device="cuda")
    for which, scale in enumerate(_scales(case)):
        src, to = (v[:, :, which], out[:, :, which]) if case["block_first"] else (v[:, which], out[:, which])
        to.copy_((src / scale).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def _values(s, t, scale):
    """What the cache's bytes stand for, in 32 bits: [..., head, dim]."""
    if s["case"]["kv"] == "4":
        return _from_fp4(s["case"], t)
    return t.view(torch.float8_e4m3fn).float() * scale if s["case"]["kv"] == "8" else t.float()


def _prepare_cache(s, lens, g, rng):
    """A cache whose requests hold `lens` tokens, a direction per head that some keys have much of, and that direction."""
    case = s["case"]
    heads, dim = case["heads"], case["dim"]
    present = _present(case, lens)
    n_blocks = int(present.sum()) + int(present.sum()) // 4 + 3
    s["n_blocks"] = n_blocks
    s["table"] = _table(rng, present, n_blocks)
    s["lens"] = torch.from_numpy(lens.astype(np.int32)).cuda()
    s["cache"] = _new_values(case, n_blocks, g)
    look = torch.empty((heads, dim), device="cuda").normal_(generator=g)
    much = torch.empty((n_blocks, case["tokens"], heads, 1), dtype=_type(case), device="cuda").exponential_(4.0, generator=g)
    _planes(s, 0).add_(much * look.to(_type(case)))
    s["cache"] = _to_cache_type(case, s["cache"])
    if case["stale"]:       # rows behind a request's last token hold anything
        rows = torch.zeros((n_blocks, case["tokens"]), dtype=torch.bool, device="cuda")
        end = torch.from_numpy(lens).cuda()
        last = (end - 1).clamp(min=0) // case["tokens"]
        ids = s["table"].long().gather(1, last[:, None])[:, 0]
        there = (ids >= 0) & (end > 0)
        behind = torch.arange(case["tokens"], device="cuda")[None] >= (end - last * case["tokens"])[:, None]
        rows[ids[there]] = behind[there]
        for which in (0, 1):
            plane = _planes(s, which)
            plane.masked_fill_(rows.view(rows.shape + (1,) * (plane.dim() - 2)), float("nan") if case["kv"] == "16" else 255)
    return look


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {"case": dict(case)}
    heads, dim, n = case["heads"], case["dim"], case["n_seqs"]
    q_heads = heads * case["group"]
    if case["op"] in ("attend", "rows"):
        if case["op"] == "attend":
            lens, rows = _lengths(case, case["longest"]), n
            s["mass"] = None
        else:
            new, lens = _counts(case)
            rows = int(new.sum()) + case["behind"]
            s["starts"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
            # where the plain form finds each row's request and its place among that one's rows
            s["n_new"], s["most"] = int(new.sum()), int(new.max())
            s["seq"] = torch.from_numpy(np.repeat(np.arange(n), new)).cuda()
            s["at"] = torch.from_numpy(np.concatenate([np.arange(m) for m in new])).cuda()
            s["new"] = torch.from_numpy(new).cuda()
        look = _prepare_cache(s, lens, g, rng)
        q = torch.empty((rows, heads, case["group"], dim), device="cuda").normal_(generator=g) + 0.7 * look[:, None]
        s["q"] = q.reshape(rows, q_heads, dim).to(_type(case))
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((rows, q_heads), device="cuda") if case["lse"] else None
        if case["op"] == "attend" and case["mass"]:
            s["mass"] = torch.empty(s["table"].shape, device="cuda").exponential_(1.0, generator=g)
        s["mass_out"] = torch.empty_like(s["mass"]) if s.get("mass") is not None else None
        return s
    # put: `new` tokens of each request (fewer for some) behind what it holds already
    new, past = _put_counts(case)
    rows = int(new.sum()) + case["behind"]
    lens = past + new
    present = np.arange(int(_blocks(lens, case["tokens"]).max()))[None] < _blocks(lens, case["tokens"])[:, None]
    # the pages that the new tokens lie in; those before them are somebody else's business here
    touched = present & (np.arange(present.shape[1])[None] >= (past // case["tokens"])[:, None])
    s["n_blocks"] = int(touched.sum()) + 5
    s["table"] = _table(rng, touched, s["n_blocks"])
    s["lens"] = torch.from_numpy(lens.astype(np.int32)).cuda()
    s["starts"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    s["one_each"], s["n_new"] = case["new"] == 1 and not case["behind"], int(new.sum())
    s["cache"] = _to_cache_type(case, _new_values(case, s["n_blocks"], g))
    # one product gave q, k and v side by side
    qkv = torch.empty((rows, q_heads + 2 * heads, dim), dtype=_type(case), device="cuda").normal_(generator=g)
    s["q"], s["k"], s["v"] = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
    s["q_out"] = torch.zeros((rows, q_heads, dim), dtype=_type(case), device="cuda")
    # where each row stands: its place in the request, or for images its time, row and column
    at = np.concatenate([np.arange(a, a + b) for a, b in zip(past, new)] + [np.zeros(case["behind"], np.int64)])
    pos = at[None] if case["axes"] == 1 else np.stack([at, at // 7 + rng.integers(0, 50, at.size), at % 97 + 3])
    s["positions"] = torch.from_numpy(pos.astype(np.int32)).cuda()
    theta = 500000.0 * (1 + seed % 7)
    s["inv_freq"] = (theta ** -(torch.arange(case["rot"] // 2, dtype=torch.float64) * 2 / case["rot"])).float().cuda()
    # learned weights of the norms, around 1
    s["weights"] = [1 + 0.3 * torch.empty(dim, device="cuda").normal_(generator=g) for _ in range(2)] if case["norm"] else None
    # where the plain form finds each row's request, page and place in it
    seq = np.repeat(np.arange(n), new)
    s["seq"] = torch.from_numpy(seq).cuda()
    s["cell"] = torch.from_numpy(at[:s["n_new"]]).cuda()
    # the two numbers of each byte of a 4-bit cache
    two = torch.tensor([[v[b & 15], v[b >> 4]] for v in (VALUES + tuple(-x for x in VALUES),) for b in range(256)])
    s["pairs"] = two.to(torch.float8_e4m3fn).cuda().view(torch.int16)[:, 0].contiguous()
    return s


EPS = 1e-6  # of the norms


# ---- one pass -------------------------------------------------------------------------------------

def _held_plain(s):
    """Keys and values of every request's places, [request, token, head, dim], 0 where there are none, and which there are."""
    c, ids = s["case"], s["table"].long()
    n, p = c["n_seqs"], c["tokens"]
    at = torch.arange(ids.shape[1] * p, device="cuda")
    seen = (at[None] < s["lens"][:, None]) & (ids >= 0).repeat_interleave(p, dim=1)
    k, v = (_values(s, _planes(s, which)[ids.clamp(min=0)], scale).reshape(n, -1, c["heads"], c["dim"])
            for which, scale in enumerate(_scales(c)))
    none = torch.zeros((), device="cuda")
    return torch.where(seen[:, :, None, None], k, none), torch.where(seen[:, :, None, None], v, none), seen


def _weights_plain(scores, seen):
    """softmax over the last axis of those that are seen, its log of the sum; nothing: weights of 0."""
    scores = torch.where(seen, scores, torch.full((), -math.inf, device="cuda"))
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(scores.sub_(top))
    total = e.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), torch.full_like(top, -math.inf))[..., 0]
    return e.div_(torch.where(total > 0, total, torch.ones_like(total))), lse


def _attend_plain(s):
    c = s["case"]
    n, dim = c["n_seqs"], c["dim"]
    k, v, seen = _held_plain(s)
    q = s["q"].float().reshape(n, c["heads"], c["group"], dim)
    scores = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(dim))
    w, lse = _weights_plain(scores, seen[:, None, None])
    got = {"out": torch.matmul(w, v.permute(0, 2, 1, 3).contiguous()).reshape(n, -1, dim).to(s["q"].dtype)}
    if c["lse"]:
        got["lse"] = lse.reshape(n, -1)
    if c["mass"]:
        got["mass"] = s["mass"] + w.sum((1, 2)).reshape(n, -1, c["tokens"]).sum(-1)
    return got


def _rows_plain(s):
    c, m, most = s["case"], s["n_new"], s["most"]
    n, heads, group, dim = c["n_seqs"], c["heads"], c["group"], c["dim"]
    k, v, seen = _held_plain(s)
    # the rows of each request side by side: [request, head, row * group, dim]
    q = torch.zeros((n, max(1, most), heads, group, dim), device="cuda")
    q[s["seq"], s["at"]] = s["q"][:m].float().reshape(m, heads, group, dim)
    q = q.permute(0, 2, 1, 3, 4).reshape(n, heads, -1, dim)
    scores = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(1.0 / math.sqrt(dim))
    seen = seen[:, None, None]
    if c["causal"]:
        upto = (s["lens"].long() - s["new"])[:, None] + 1 + torch.arange(max(1, most), device="cuda")
        seen = seen & (torch.arange(seen.shape[-1], device="cuda") < upto.repeat_interleave(group, dim=1)[:, None, :, None])
    w, lse = _weights_plain(scores, seen)
    out = torch.matmul(w, v.permute(0, 2, 1, 3).contiguous()).reshape(n, heads, -1, group, dim).permute(0, 2, 1, 3, 4)
    s["out"][:m] = out[s["seq"], s["at"]].reshape(m, heads * group, dim).to(s["out"].dtype)
    got = {"out": s["out"]}
    if c["lse"]:
        s["lse"][:m] = lse.reshape(n, heads, -1, group).permute(0, 2, 1, 3)[s["seq"], s["at"]].reshape(m, heads * group)
        got["lse"] = s["lse"]
    return got


def _normed(x, weight):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight


def _rotated(c, x, cos, sin):
    """x [row, head, dim] in 32 bits, its first `rot` dimensions turned pair by pair."""
    r = c["rot"]
    cos, sin = cos[:, None], sin[:, None]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _put_plain(s):
    c, n = s["case"], s["n_new"]
    sections = torch.tensor(_sections(c), device="cuda")
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), sections, output_size=c["rot"] // 2)
    angle = s["positions"][:, :n].double()[axis].t() * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    page = s["table"].long()[s["seq"], s["cell"] // c["tokens"]]
    q, k, v = s["q"][:n].float(), s["k"][:n].float(), s["v"][:n].float()
    if c["norm"]:
        q, k = _normed(q, s["weights"][0]), _normed(k, s["weights"][1])
    for which, x in enumerate((_rotated(c, k, cos, sin), v)):
        x = _to_fp4(c, x) if c["kv"] == "4" else x.to(s["cache"].dtype)
        _planes(s, which)[page, s["cell"] % c["tokens"]] = x
    s["q_out"][:n] = _rotated(c, q, cos, sin).to(s["q_out"].dtype)
    return _put_shown(s)


def _put_shown(s):
    """The cache and q.  A cache in 4 bits as its numbers, in a type of 8 bits that holds them, and the powers of 2 that they
    are multiplied with."""
    if s["case"]["kv"] == "16":
        return {"cache": s["cache"], "q": s["q_out"]}
    n = s["case"]["heads"] * s["case"]["dim"] // 2
    pairs = torch.index_select(s["pairs"], 0, s["cache"][..., :n].int().flatten())
    return {"numbers": pairs.view(torch.float8_e4m3fn), "powers": s["cache"][..., n:].view(torch.float8_e8m0fnu), "q": s["q_out"]}


def _decoder(s):
    """The handle that a program makes once for its cache, and keeps."""
    from paper_2601_20309_amd import binding as B, decode as D, workloads as W
    c = s["case"]
    head = D.fp4_head_bytes(c["dim"]) if c["kv"] == "4" else c["dim"]
    shape = W.KVShape(c["layers"], c["heads"], head, c["tokens"], s["n_blocks"], 1, 2 if c["kv"] == "16" else 1)
    if c["op"] == "put":
        s["rope"] = D.Rope(s["inv_freq"], _sections(c), interleaved=c["interleaved"])
        s["norm"] = D.HeadNorm(s["weights"][0], s["weights"][1], EPS) if c["norm"] else None
    cfg = B.make_config(shape, hbm_layout=B.KV_HBM_BLOCK_FIRST if c["block_first"] else B.KV_HBM_LAYER_FIRST)
    k_scale, v_scale = _scales(c)
    x = B.KV_FP16 if c["x"] == "fp16" else B.KV_BF16
    return D.Decoder(cfg, s["cache"].data_ptr(), n_heads=c["heads"] * c["group"], x_type=x,
                     kv_type={"16": x, "8": B.KV_FP8, "4": B.KV_FP4}[c["kv"]], k_scale=k_scale, v_scale=v_scale,
                     max_seqs=c["n_seqs"], max_blocks=s["table"].shape[1], weigh=bool(c.get("mass")),
                     max_rows=s["q"].shape[0] if c["op"] == "rows" else 0)


def _ok(rc):
    if rc != 0:
        raise RuntimeError("refused: %d" % rc)


def _run_own(s):
    c = s["case"]
    d = s.get("decoder")
    if d is None:
        d = s["decoder"] = _decoder(s)
    layer = c["layers"] - 1
    if c["op"] == "put":
        _ok(d.kv_put(layer, s["k"], s["v"], s["table"], s["lens"], q=s["q"], q_out=s["q_out"],
                     starts=None if s["one_each"] else s["starts"], rope=s["rope"], positions=s["positions"], norm=s["norm"]))
        return _put_shown(s)
    if c["op"] == "rows":
        _ok(d.kv_attend_rows(layer, s["q"], s["table"], s["lens"], s["out"], starts=s["starts"], causal=c["causal"], lse=s["lse"]))
        return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}
    _ok(d.kv_attend(layer, s["q"], s["table"], s["lens"], s["out"], lse=s["lse"], mass=s["mass"], mass_out=s["mass_out"]))
    got = {"out": s["out"]}
    if c["lse"]:
        got["lse"] = s["lse"]
    if c["mass"]:
        got["mass"] = s["mass_out"]
    return got


def run(s):
    if own:
        return _run_own(s)
    return {"rows": _rows_plain, "attend": _attend_plain, "put": _put_plain}[s["case"]["op"]](s)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    """Every key and value that is attended to, and every new row, in and out once; the products that are not masked."""
    heads, q_heads, dim, n = case["heads"], case["heads"] * case["group"], case["dim"], case["n_seqs"]
    if case["op"] == "put":
        rows = int(_put_counts(case)[0].sum())
        return {"bytes": rows * (4 * dim * (q_heads + heads) + 2 * _token_bytes(case)),
                "flops": rows * (q_heads + heads) * (case["rot"] * 3 + (4 * dim if case["norm"] else 0))}
    new, lens = (1, _lengths(case, case["longest"])) if case["op"] == "attend" else _counts(case)
    held = _in_blocks(case, lens)
    rows = n if case["op"] == "attend" else int(new.sum())
    extra = 8 * int(_blocks(lens, case["tokens"]).sum()) if case.get("mass") else 0
    extra += 4 * rows * q_heads if case["lse"] else 0
    if case["op"] == "rows" and case["causal"]:
        pairs = 0       # (row, token that it sees)
        for i in range(n):
            upto = np.cumsum(np.concatenate([[0], held[i]]))
            place = np.arange(lens[i] - new[i], lens[i])
            block, inside = (place + 1) // case["tokens"], (place + 1) % case["tokens"]
            there = np.concatenate([held[i] > 0, [False]])
            pairs += int((upto[block] + inside * there[np.minimum(block, there.size - 1)]).sum())
    else:
        pairs = int((held.sum(1) * new).sum())
    used = held[np.asarray(new) > 0] if case["op"] == "rows" else held
    return {"bytes": int(used.sum()) * 2 * _token_bytes(case) + 4 * rows * q_heads * dim + extra, "flops": 4 * pairs * q_heads * dim}


# ---- the same from the definitions, in 64 bits ----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_put(s, case) if case["op"] == "put" else _exact_attend(s, case)


def _wide(case, x, which):
    """A token's bytes as the numbers that they stand for: x [token, ...] to [token, head, dim] in 64 bits."""
    heads, dim = case["heads"], case["dim"]
    if case["kv"] == "8":
        return x.view(torch.float8_e4m3fn).to(torch.float64) * _scales(case)[which]
    if case["kv"] == "16":
        return x.to(torch.float64)
    n = heads * dim // 2
    power = torch.exp2(x[:, n:].double() - 127).reshape(-1, heads, dim // 32, 1)
    out = torch.empty((x.shape[0], heads * dim), dtype=torch.float64, device="cuda")
    for half in (0, 1):
        code = (x[:, :n] >> (4 * half)) & 15
        e, odd = ((code >> 1) & 3).double(), (code & 1).double()
        size = torch.where(e == 0, odd * 0.5, (1 + odd / 2) * torch.exp2(e - 1))
        out[:, half::2] = torch.where(code >= 8, -size, size)
    return (out.reshape(-1, heads, dim // 32, 32) * power).reshape(-1, heads, dim)


def _exact_attend(s, case):
    p, g, dim, n = case["tokens"], case["group"], case["dim"], case["n_seqs"]
    table, lens = s["table"].cpu().numpy(), s["lens"].cpu().numpy().astype(np.int64)
    starts = s["starts"].cpu().numpy() if case["op"] == "rows" else np.arange(n + 1)
    out, lse = s["out"].double(), torch.zeros((s["q"].shape[0], case["heads"] * g), dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if case.get("mass") else None
    for i in range(n):
        a, b = int(starts[i]), int(starts[i + 1])
        t = np.arange(lens[i])
        t = t[table[i, t // p] >= 0]
        lse[a:b] = -math.inf
        if a == b or not t.size:
            continue
        page, row = (torch.from_numpy(x.astype(np.int64)).cuda() for x in (table[i, t // p], t % p))
        k, v = (_wide(case, _planes(s, which)[page, row], which) for which in (0, 1))
        place = torch.from_numpy(t).cuda()
        if case["op"] == "rows" and case["causal"]:
            unseen = place[None] > torch.arange(int(lens[i]) - (b - a), int(lens[i]), device="cuda")[:, None]
        else:
            unseen = torch.zeros((b - a, t.size), dtype=torch.bool, device="cuda")
        for h in range(case["heads"]):
            keys, values = k[:, h].t().contiguous(), v[:, h].contiguous()
            for j in range(h * g, (h + 1) * g):
                x = (s["q"][a:b, j].double() @ keys) / math.sqrt(dim)
                x[unseen] = -math.inf
                lse[a:b, j] = torch.logsumexp(x, 1)
                w = torch.exp(x - lse[a:b, j, None]).nan_to_num(0.0)
                out[a:b, j] = w @ values
                if mass is not None:
                    mass[i].index_add_(0, place // p, w.sum(0))
    got = {"out": out}
    if case["lse"]:
        got["lse"] = lse
    if mass is not None:
        got["mass"] = mass
    return got


def _exact_put(s, case):
    n, r, p = s["n_new"], case["rot"], case["tokens"]
    pos, freq = s["positions"].cpu().numpy().astype(np.float64), s["inv_freq"].cpu().numpy().astype(np.float64)
    axis_of = [a for a, k in enumerate(_sections(case)) for _ in range(k)]
    turn = np.exp(1j * np.stack([pos[a, :n] * f for a, f in zip(axis_of, freq)], 1))        # [row, pair]
    turn = torch.from_numpy(turn).cuda()[:, None]

    def spin(x, which):
        x = x[:n].double().clone()
        if case["norm"]:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / case["dim"] + EPS) * s["weights"][which].double()
        one, two = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(x[..., one], x[..., two]) * turn
        x[..., one], x[..., two] = z.real, z.imag
        return x

    table, cell, seq = (s[k].cpu().numpy() for k in ("table", "cell", "seq"))
    page = torch.from_numpy(table[seq, cell // p].astype(np.int64)).cuda()
    row = torch.from_numpy(cell % p).cuda()
    at = case["layers"] - 1
    q = s["q_out"].double()
    q[:n] = spin(s["q"], 0)
    new = (spin(s["k"], 1), s["v"][:n].double())
    plane = lambda x, which: x[:, at, which] if case["block_first"] else x[at, which]  # noqa: E731
    if case["kv"] == "16":
        cache = s["cache"].to(torch.float64)
        for which, x in enumerate(new):
            plane(cache, which)[page, row] = x
        return {"cache": cache, "q": q}
    # what was there, and of the new tokens 32 dimensions at a time: the power of 2 that brings the largest to 4 or more and under 8,
    # and the number nearest to each quotient
    half = case["heads"] * case["dim"] // 2
    shown = _put_shown(s)
    numbers = shown["numbers"].double().reshape(s["cache"].shape[:-1] + (2 * half,))
    powers = shown["powers"].double()
    low, high = (2.0 ** -23, 2.0 ** 13) if case["x"] == "fp16" else (2.0 ** -126, 2.0 ** 125)
    near = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    for which, x in enumerate(new):
        g = x.reshape(n, -1, 32)
        power = torch.exp2(torch.floor(torch.log2(g.abs().amax(-1).clamp(min=2.0 ** -200))) - 2).clamp(low, high)
        off = ((g.abs() / power[..., None])[..., None] - near).abs()
        # of two that are as near the one at an even place
        off[..., 1::2] = torch.where(off[..., 1::2] == off.amin(-1, keepdim=True), off[..., 1::2] * (1 + 2.0 ** -40), off[..., 1::2])
        number = near[off.argmin(-1)]
        plane(numbers, which)[page, row] = torch.where(torch.signbit(g), -number, number).reshape(n, -1)
        plane(powers, which)[page, row] = power
    return {"numbers": numbers.flatten(), "powers": powers, "q": q}
