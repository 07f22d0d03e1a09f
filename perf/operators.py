"""The operators of a decode step over the paged KV cache, as cases that can be timed and compared.

  put     new tokens' q and k get their rotary positions, k and v go into their pages
  attend  one new token of every request over the pages it holds
  evict   the blocks that attention has weighed least leave a request

Where `own` is false, `run` computes them from elementary torch operations in 32
bits, rounded once at the end; where it is true, through the package's decoder.
Shapes are those of the workloads module, their shards under tensor parallelism,
and generic ones that are a power of two nowhere.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}


def _attend(n_seqs, longest, heads, group, dim, tokens, **opt):
    c = dict(op="attend", n_seqs=n_seqs, longest=longest, heads=heads, group=group, dim=dim, tokens=tokens,
             type="bf16", spread="lognormal", mass=False, lse=False, holes=0.0, stale=False, layers=1,
             block_first=False, shape_seed=1)
    c.update(opt)
    return c


def _put(n_seqs, new, past, heads, group, dim, tokens, **opt):
    c = dict(op="put", n_seqs=n_seqs, new=new, past=past, heads=heads, group=group, dim=dim, tokens=tokens,
             type="bf16", axes=1, rot=dim, interleaved=False, fused=True, behind=0, layers=1, block_first=False,
             shape_seed=1)
    c.update(opt)
    return c


def _evict(n_seqs, longest, budget, first, last, tokens, **opt):
    c = dict(op="evict", n_seqs=n_seqs, longest=longest, budget=budget, first=first, last=last, tokens=tokens,
             spread="lognormal", cap=longest, shape_seed=1)
    c.update(opt)
    return c


def listed():
    named = {
        # the smallest attention there is a configuration for: a few short requests, all latency
        "attend_tiny": _attend(3, 100, 2, 2, 64, 16, layers=2),
        # a serving batch of Llama-3-8B-shaped requests (median 1024, up to 8192 tokens), weights kept for eviction
        "attend_batch": _attend(32, 8192, 8, 4, 128, 16, mass=True),
        # the 70B-shaped long context: 4 requests of 32768 tokens in blocks of 32
        "attend_long_70b": _attend(4, 32768, 8, 8, 128, 32, spread="equal"),
        # one of eight tensor-parallel shards and one request alone: what cannot be split over heads or requests
        "attend_one_request_shard": _attend(1, 131072, 1, 8, 128, 16, spread="equal", lse=True),
        # a large batch whose cache is held in 8 bits
        "attend_fp8_batch": _attend(128, 4096, 8, 5, 128, 16, type="fp8", block_first=True),
        # blocks of 5 tokens, 3 heads of 40, pages that are not there, requests of no and of one token, NaN behind the ends
        "attend_ragged": _attend(37, 1700, 3, 3, 40, 5, type="fp16", spread="ragged", mass=True, lse=True, holes=0.1,
                                 stale=True, layers=2),
        # a decode step of 64 requests: one token each, far into their contexts
        "put_decode": _put(64, 1, 30000, 8, 4, 128, 16, layers=2),
        # prompts with images: 3 axes, 8192 tokens in all
        "put_prompts_3_axes": _put(4, 2048, 0, 8, 4, 128, 16, axes=3),
        # half of each head rotates, neighbours paired, an 8-bit cache in blocks of 5, rows of padding behind
        "put_ragged_fp8": _put(7, 300, 900, 3, 4, 80, 5, type="fp8", rot=40, interleaved=True, behind=61),
        # a serving batch at its budget of 2048 tokens, 8192 at most
        "evict_batch": _evict(64, 512, 128, 1, 4, 16),
        # a few very long requests: 131072 tokens in blocks of 16, a quarter stays
        "evict_long": _evict(8, 8192, 2048, 4, 32, 16, spread="equal"),
    }
    return [dict(c, name=n) for n, c in named.items()]


def draw(rng):
    pick = rng.choice
    logu = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = pick(["attend", "attend", "attend", "put", "put", "evict"])
    common = dict(shape_seed=rng.randrange(1 << 30))
    if op == "evict":
        longest = logu(2, 8192)
        n_seqs = max(1, min(logu(1, 256), 65536 // longest))
        return _evict(n_seqs, longest, max(1, int(longest * rng.uniform(0.1, 0.9))), rng.randrange(0, 5),
                      1 + logu(1, 33), pick([5, 16, 16, 32]), spread=pick(["lognormal", "equal", "ragged"]),
                      cap=pick([longest, longest, max(1, longest // 3)]), **common)
    heads, group = pick([(8, 4), (8, 4), (8, 8), (8, 5), (1, 4), (1, 8), (2, 2), (4, 7), (3, 3), (2, 16), (1, 24)])
    dim = pick([128, 128, 128, 64, 40, 80, 96, 192, 256])
    common.update(type=pick(["bf16", "bf16", "fp16", "fp8"]), tokens=pick([16, 16, 16, 32, 8, 5, 24]),
                  layers=pick([1, 2]), block_first=pick([False, False, True]))
    if op == "attend":
        row = 2 * heads * dim * 2 * common["layers"]
        longest = logu(1, 131072)
        most = min((400 << 20) // row, (1 << 30) // (heads * group * dim))      # tokens of a case
        longest = min(longest, most)
        n_seqs = max(1, min(logu(1, 200), most // longest))
        return _attend(n_seqs, longest, heads, group, dim, common.pop("tokens"),
                       spread=pick(["lognormal", "equal", "ragged"]), mass=pick([False, True]), lse=pick([False, True]),
                       holes=pick([0.0, 0.0, 0.05]), stale=pick([False, True]), **common)
    n_seqs = logu(1, 128)
    new = pick([1, 1, logu(2, max(3, min(8192, (32 << 20) // (heads * group * dim)) // n_seqs))])
    axes = pick([1, 1, 3])
    return _put(n_seqs, new, pick([0, logu(1, 4000), logu(4000, 120000)]), heads, group, dim, common.pop("tokens"),
                axes=axes, rot=pick([dim, dim, dim // 16 * 8]), interleaved=pick([False, True]), fused=pick([True, False]),
                behind=pick([0, 0, 13]), **common)


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


def _blocks(lens, tokens):
    return -(-lens // tokens)


def _present(case, lens):
    """Which entries of the requests' tables name a page: [request, entry]."""
    held = _blocks(lens, case["tokens"])
    at = np.arange(max(1, int(held.max())))[None] < held[:, None]
    if case.get("holes"):
        at &= np.random.default_rng(case["shape_seed"] + 1).random(at.shape) >= case["holes"]
    return at


def _attended(case, lens):
    """Tokens that are attended to: those of present pages."""
    at, p = _present(case, lens), case["tokens"]
    in_block = np.clip(lens[:, None] - np.arange(at.shape[1])[None] * p, 0, p)
    return int((in_block * at).sum())


def _sections(case):
    """Pairs of each axis: time, height, width in about 1 : 1.5 : 1.5."""
    pairs = case["rot"] // 2
    if case["axes"] == 1:
        return (pairs,)
    t = pairs // 4
    h = (pairs - t) // 2
    return (t, h, pairs - t - h)


def _type(case):
    """Of q, k, v and the outputs; a cache in 8 bits goes with bf16."""
    return torch.float16 if case["type"] == "fp16" else torch.bfloat16


def _scales(case):
    return (0.03, 0.0125) if case["type"] == "fp8" else (1.0, 1.0)


def _x_bytes(case):
    return 1 if case["type"] == "fp8" else 2


# ---- inputs ---------------------------------------------------------------------------------------

def _table(rng, present, n_blocks):
    table = np.full(present.shape, -1, np.int32)
    table[present] = rng.permutation(n_blocks)[:int(present.sum())]
    return torch.from_numpy(table).cuda()


def _planes(s, which):
    """K (0) or V (1) of the case's layer: [block, token, head, dim], in the cache's own bytes."""
    c, cache = s["case"], s["cache"]
    at = c["layers"] - 1
    return cache[:, at, which] if c["block_first"] else cache[at, which]


def _new_cache(case, n_blocks, g):
    """A cache of N(0, 1) in the 16-bit type."""
    inner = (case["tokens"], case["heads"], case["dim"])
    dims = (n_blocks, case["layers"], 2) + inner if case["block_first"] else (case["layers"], 2, n_blocks) + inner
    return torch.empty(dims, dtype=_type(case), device="cuda").normal_(generator=g)


def _to_cache_type(case, v):
    """Values of the 16-bit type as the cache holds them; K and V have one scale each."""
    if case["type"] != "fp8":
        return v
    out = torch.empty(v.shape, dtype=torch.uint8, device="cuda")
    for which, scale in enumerate(_scales(case)):
        src, to = (v[:, :, which], out[:, :, which]) if case["block_first"] else (v[:, which], out[:, which])
        to.copy_((src / scale).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {"case": dict(case)}
    if case["op"] == "evict":
        held = _lengths(case, case["longest"])
        p = case["tokens"]
        lens = np.maximum(held * p - np.random.default_rng(case["shape_seed"] + 2).integers(0, p, held.size), 0) * (held > 0)
        present = np.arange(case["longest"])[None] < held[:, None]
        s["n_blocks"] = int(present.sum()) + 7
        s["table"] = _table(rng, present, s["n_blocks"])
        s["lens"] = torch.from_numpy(lens.astype(np.int32)).cuda()
        # heavy-tailed, some of it in steps that several blocks share, none yet for the newest
        mass = torch.empty(present.shape, device="cuda").log_normal_(0.0, 2.0, generator=g)
        mass[:, ::3] = torch.round(mass[:, ::3] * 4) / 4
        at = torch.arange(case["longest"], device="cuda")[None]
        s["mass"] = torch.where(at < torch.from_numpy(held).cuda()[:, None] - 2, mass, torch.zeros_like(mass))
        s["table_out"], s["lens_out"], s["mass_out"] = (torch.empty_like(s[k]) for k in ("table", "lens", "mass"))
        n, cap = case["n_seqs"], case["cap"]
        s["ids"], s["at"] = (torch.empty((n, cap), dtype=torch.int32, device="cuda") for _ in range(2))
        s["count"] = torch.empty(n, dtype=torch.int32, device="cuda")
        return s
    heads, dim, n = case["heads"], case["dim"], case["n_seqs"]
    q_heads = heads * case["group"]
    if case["op"] == "attend":
        lens = _lengths(case, case["longest"])
        present = _present(case, lens)
        n_blocks = int(present.sum()) + int(present.sum()) // 4 + 3
        s["table"] = _table(rng, present, n_blocks)
        s["lens"] = torch.from_numpy(lens.astype(np.int32)).cuda()
        v = _new_cache(case, n_blocks, g)
        # what attention looks for: a direction per head that queries share and some keys have much of
        look = torch.empty((heads, dim), device="cuda").normal_(generator=g)
        s["cache"] = v
        much = torch.empty((n_blocks, case["tokens"], heads, 1), dtype=v.dtype, device="cuda").exponential_(4.0, generator=g)
        _planes(s, 0).add_(much * look.to(v.dtype))
        q = torch.empty((n, heads, case["group"], dim), device="cuda").normal_(generator=g) + 0.7 * look[:, None]
        s["q"] = q.reshape(n, q_heads, dim).to(_type(case))
        if case["stale"]:       # rows behind a request's last token hold anything
            rows = torch.zeros((n_blocks, case["tokens"]), dtype=torch.bool, device="cuda")
            end = torch.from_numpy(lens).cuda()
            last = (end - 1).clamp(min=0) // case["tokens"]
            ids = s["table"].long().gather(1, last[:, None])[:, 0]
            there = (ids >= 0) & (end > 0)
            behind = torch.arange(case["tokens"], device="cuda")[None] >= (end - last * case["tokens"])[:, None]
            rows[ids[there]] = behind[there]
            for which in (0, 1):
                _planes(s, which).masked_fill_(rows[:, :, None, None], float("nan"))
        s["cache"] = _to_cache_type(case, v)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((n, q_heads), device="cuda") if case["lse"] else None
        s["mass"] = torch.empty(present.shape, device="cuda").exponential_(1.0, generator=g) if case["mass"] else None
        s["mass_out"] = torch.empty_like(s["mass"]) if case["mass"] else None
        return s
    # put: `new` tokens of each request (fewer for some) behind what it holds already
    few = np.random.default_rng(case["shape_seed"])
    new = np.full(n, case["new"]) if case["new"] == 1 else few.integers((case["new"] + 1) // 2, case["new"] + 1, n)
    past = few.integers(case["past"] // 2, case["past"] + 1, n)
    rows = int(new.sum()) + case["behind"]
    lens = past + new
    present = np.arange(int(_blocks(lens, case["tokens"]).max()))[None] < _blocks(lens, case["tokens"])[:, None]
    # the pages that the new tokens lie in; those before them are somebody else's business here
    touched = present & (np.arange(present.shape[1])[None] >= (past // case["tokens"])[:, None])
    n_blocks = int(touched.sum()) + 5
    s["table"] = _table(rng, touched, n_blocks)
    s["lens"] = torch.from_numpy(lens.astype(np.int32)).cuda()
    s["starts"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    s["one_each"], s["n_new"] = case["new"] == 1 and not case["behind"], int(new.sum())
    s["cache"] = _to_cache_type(case, _new_cache(case, n_blocks, g))
    if case["fused"]:           # one product gave q, k and v side by side
        qkv = torch.empty((rows, q_heads + 2 * heads, dim), dtype=_type(case), device="cuda").normal_(generator=g)
        s["q"], s["k"], s["v"] = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
    else:
        s["q"], s["k"], s["v"] = (torch.empty((rows, h, dim), dtype=_type(case), device="cuda").normal_(generator=g)
                                  for h in (q_heads, heads, heads))
    s["q_out"] = torch.zeros((rows, q_heads, dim), dtype=_type(case), device="cuda")
    # where each row stands: its place in the request, or for images its time, row and column
    at = np.concatenate([np.arange(a, a + b) for a, b in zip(past, new)] + [np.zeros(case["behind"], np.int64)])
    pos = at[None] if case["axes"] == 1 else np.stack([at, at // 7 + rng.integers(0, 50, at.size), at % 97 + 3])
    s["positions"] = torch.from_numpy(pos.astype(np.int32)).cuda()
    theta = 500000.0 * (1 + seed % 7)
    s["inv_freq"] = (theta ** -(torch.arange(case["rot"] // 2, dtype=torch.float64) * 2 / case["rot"])).float().cuda()
    # where the plain form finds each row's request, page and place in it
    seq = np.repeat(np.arange(n), new)
    s["seq"] = torch.from_numpy(seq).cuda()
    s["cell"] = torch.from_numpy(at[:s["n_new"]]).cuda()
    return s


# ---- one pass -------------------------------------------------------------------------------------

def _values(s, t, scale):
    """What the cache's bytes stand for, in 32 bits."""
    if s["case"]["type"] == "fp8":
        return t.view(torch.float8_e4m3fn).float() * scale
    return t.float()


def _attend_plain(s):
    c = s["case"]
    n, heads, dim, p = c["n_seqs"], c["heads"], c["dim"], c["tokens"]
    ids = s["table"].long()
    at = torch.arange(ids.shape[1] * p, device="cuda")
    seen = (at[None] < s["lens"][:, None]) & (ids >= 0).repeat_interleave(p, dim=1)
    k, v = (_values(s, _planes(s, which)[ids.clamp(min=0)], scale).reshape(n, -1, heads, dim)
            for which, scale in enumerate(_scales(c)))
    none = torch.zeros((), device="cuda")
    k, v = torch.where(seen[:, :, None, None], k, none), torch.where(seen[:, :, None, None], v, none)
    q = s["q"].float().reshape(n, heads, c["group"], dim)
    scores = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(dim))
    scores = torch.where(seen[:, None, None], scores, torch.full((), -math.inf, device="cuda"))
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(scores - top)
    total = e.sum(-1, keepdim=True)
    w = e / torch.where(total > 0, total, torch.ones_like(total))
    out = torch.matmul(w, v.permute(0, 2, 1, 3).contiguous())
    got = {"out": out.reshape(n, -1, dim).to(s["q"].dtype)}
    if c["lse"]:
        got["lse"] = torch.where(total > 0, top + torch.log(total), torch.full_like(top, -math.inf)).reshape(n, -1)
    if c["mass"]:
        got["mass"] = s["mass"] + w.sum((1, 2)).reshape(n, -1, p).sum(-1)
    return got


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
    for which, x in enumerate((_rotated(c, s["k"][:n].float(), cos, sin), s["v"][:n].float())):
        if c["type"] == "fp8":
            x = (x / _scales(c)[which]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        _planes(s, which)[page, s["cell"] % c["tokens"]] = x.to(s["cache"].dtype)
    s["q_out"][:n] = _rotated(c, s["q"][:n].float(), cos, sin).to(s["q_out"].dtype)
    return {"cache": _shown(s), "q": s["q_out"]}


def _shown(s):
    return s["cache"].view(torch.float8_e4m3fn) if s["case"]["type"] == "fp8" else s["cache"]


def _evict_plain(s):
    c, p = s["case"], s["case"]["tokens"]
    at = torch.arange(c["longest"], device="cuda")[None]
    held = ((s["lens"].long() + p - 1) // p)[:, None]
    may = (at >= c["first"]) & (at < held - c["last"])
    count = torch.minimum((held - c["budget"]).clamp(min=0), may.sum(1, keepdim=True)).clamp(max=c["cap"])
    key = torch.where(may, s["mass"], torch.full((), math.inf, device="cuda"))
    rank = torch.argsort(torch.argsort(key, dim=1, stable=True), dim=1)
    goes = may & (rank < count)
    # those that stay first, in their order; then those that go; then what holds nothing
    order = torch.argsort(goes.long() + 2 * (at >= held).long(), dim=1, stable=True)
    stays = at < held - count
    table = torch.where(stays, s["table"].gather(1, order), torch.full_like(s["table"], -1))
    mass = torch.where(stays, s["mass"].gather(1, order), torch.zeros_like(s["mass"]))
    gone = torch.argsort(goes.long(), dim=1, stable=True, descending=True)[:, :c["cap"]]
    listed_ = at[:, :c["cap"]] < count
    none = torch.full((), -1, dtype=torch.int32, device="cuda")
    return {"table": table, "mass": mass, "lens": (s["lens"] - count[:, 0] * p).to(torch.int32),
            "ids": torch.where(listed_, s["table"].gather(1, gone), none),
            "at": torch.where(listed_, gone.to(torch.int32), none), "count": count[:, 0].to(torch.int32)}


def _decoder(s):
    """The handle that a program makes once for its cache, and keeps."""
    from paper_2601_20309_amd import binding as B, decode as D, workloads as W
    c = s["case"]
    if c["op"] == "evict":
        shape = W.KVShape(1, 1, 8, c["tokens"], s["n_blocks"], 1)
        cache = s["cache"] = torch.empty(shape.cache_dims(), dtype=torch.bfloat16, device="cuda")
    else:
        cache = s["cache"]
        shape = W.KVShape(c["layers"], c["heads"], c["dim"], c["tokens"], cache.shape[0 if c["block_first"] else 2], 1, _x_bytes(c))
        if c["op"] == "put":
            s["rope"] = D.Rope(s["inv_freq"], _sections(c), interleaved=c["interleaved"])
    cfg = B.make_config(shape, hbm_layout=B.KV_HBM_BLOCK_FIRST if c.get("block_first") else B.KV_HBM_LAYER_FIRST)
    k_scale, v_scale = _scales(c) if c["op"] != "evict" else (1.0, 1.0)
    kinds = {"bf16": B.KV_BF16, "fp16": B.KV_FP16, "fp8": B.KV_FP8}
    kv = kinds[c.get("type", "bf16")]
    return D.Decoder(cfg, cache.data_ptr(), n_heads=c.get("heads", 1) * c.get("group", 1),
                     x_type=B.KV_FP16 if kv == B.KV_FP16 else B.KV_BF16, kv_type=kv, k_scale=k_scale, v_scale=v_scale,
                     max_seqs=c["n_seqs"], max_blocks=s["table"].shape[1])


def _ok(rc):
    if rc != 0:
        raise RuntimeError("refused: %d" % rc)


def _run_own(s):
    c = s["case"]
    d = s.get("decoder")
    if d is None:
        d = s["decoder"] = _decoder(s)
    if c["op"] == "attend":
        _ok(d.kv_attend(c["layers"] - 1, s["q"], s["table"], s["lens"], s["out"], lse=s["lse"], mass=s["mass"],
                        mass_out=s["mass_out"]))
        got = {"out": s["out"]}
        if c["lse"]:
            got["lse"] = s["lse"]
        if c["mass"]:
            got["mass"] = s["mass_out"]
        return got
    if c["op"] == "put":
        _ok(d.kv_put(c["layers"] - 1, s["k"], s["v"], s["table"], s["lens"], q=s["q"], q_out=s["q_out"],
                     starts=None if s["one_each"] else s["starts"], rope=s["rope"], positions=s["positions"]))
        return {"cache": _shown(s), "q": s["q_out"]}
    _ok(d.kv_evict(s["table"], s["lens"], s["mass"], budget=c["budget"], n_first=c["first"], n_last=c["last"],
                   evicted_ids=s["ids"], evicted_at=s["at"], n_evicted=s["count"], table_out=s["table_out"],
                   lens_out=s["lens_out"], mass_out=s["mass_out"]))
    return {"table": s["table_out"], "mass": s["mass_out"], "lens": s["lens_out"], "ids": s["ids"], "at": s["at"],
            "count": s["count"]}


def run(s):
    if own:
        return _run_own(s)
    return {"attend": _attend_plain, "put": _put_plain, "evict": _evict_plain}[s["case"]["op"]](s)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    """Every key and value that is attended to, or every new row, once; the weights and tables in and out."""
    if case["op"] == "evict":
        held = _lengths(case, case["longest"])
        rows = case["n_seqs"] * case["longest"]
        return {"bytes": int(8 * held.sum() + 8 * rows + 8 * case["n_seqs"] * case["cap"]), "flops": 0}
    q_heads, dim, x = case["heads"] * case["group"], case["dim"], _x_bytes(case)
    if case["op"] == "put":
        few = np.random.default_rng(case["shape_seed"])
        n = case["n_seqs"]
        new = np.full(n, case["new"]) if case["new"] == 1 else few.integers((case["new"] + 1) // 2, case["new"] + 1, n)
        rows = int(new.sum())
        return {"bytes": rows * dim * (4 * q_heads + 2 * case["heads"] * (2 + x)),
                "flops": rows * case["rot"] * 3 * (q_heads + case["heads"])}
    lens = _lengths(case, case["longest"])
    tokens = _attended(case, lens)
    extra = 8 * int(_blocks(lens, case["tokens"]).sum()) if case["mass"] else 0
    return {"bytes": tokens * case["heads"] * dim * 2 * x + 4 * case["n_seqs"] * q_heads * dim + extra,
            "flops": 4 * tokens * q_heads * dim}


# ---- the same from the definitions, in 64 bits ----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "put": _exact_put, "evict": _exact_evict}[case["op"]](s, case)


def _exact_attend(s, case):
    p, g, dim, n = case["tokens"], case["group"], case["dim"], case["n_seqs"]
    scale = dict(zip("kv", _scales(case)))
    table, lens = s["table"].cpu().numpy(), s["lens"].cpu().numpy()
    q_heads = case["heads"] * g
    out = torch.zeros((n, q_heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((n, q_heads), -math.inf, dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if case["mass"] else None

    def wide(which, i):
        """Keys or values [token, head, dim] of request i's present pages, and each token's entry."""
        cells = [(table[i, t // p], t % p, t // p) for t in range(lens[i]) if table[i, t // p] >= 0]
        page, row, entry = (torch.tensor(v, dtype=torch.int64, device="cuda") for v in zip(*cells))
        x = _planes(s, "kv".index(which))[page, row]
        x = x.view(torch.float8_e4m3fn).to(torch.float64) * scale[which] if case["type"] == "fp8" else x.to(torch.float64)
        return x, entry

    for i in range(n):
        if not any(table[i, j] >= 0 for j in range(-(-int(lens[i]) // p))):
            continue
        k, entry = wide("k", i)
        v, _ = wide("v", i)
        for h in range(case["heads"]):
            q = s["q"][i, h * g:(h + 1) * g].double()
            a = (k[:, h] @ q.t()) / math.sqrt(dim)                  # [token, query]
            lse[i, h * g:(h + 1) * g] = torch.logsumexp(a, 0)
            w = torch.softmax(a, 0)
            out[i, h * g:(h + 1) * g] = w.t() @ v[:, h]
            if mass is not None:
                mass[i].index_add_(0, entry, w.sum(1))
    got = {"out": out}
    if case["lse"]:
        got["lse"] = lse
    if case["mass"]:
        got["mass"] = mass
    return got


def _exact_put(s, case):
    n, r, p = s["n_new"], case["rot"], case["tokens"]
    pos, freq = s["positions"].cpu().numpy().astype(np.float64), s["inv_freq"].cpu().numpy().astype(np.float64)
    axis_of = [a for a, k in enumerate(_sections(case)) for _ in range(k)]
    turn = np.exp(1j * np.stack([pos[a, :n] * f for a, f in zip(axis_of, freq)], 1))        # [row, pair]
    turn = torch.from_numpy(turn).cuda()[:, None]

    def spin(x):
        x = x[:n].double().clone()
        one, two = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(x[..., one], x[..., two]) * turn
        x[..., one], x[..., two] = z.real, z.imag
        return x

    table, cell, seq = (s[k].cpu().numpy() for k in ("table", "cell", "seq"))
    page = torch.from_numpy(table[seq, cell // p].astype(np.int64)).cuda()
    row = torch.from_numpy(cell % p).cuda()
    cache = _shown(s).to(torch.float64)
    for which, x in enumerate((spin(s["k"]), s["v"][:n].double())):
        x = (x / _scales(case)[which]).clamp(-448, 448) if case["type"] == "fp8" else x
        at = case["layers"] - 1
        plane = cache[:, at, which] if case["block_first"] else cache[at, which]
        plane[page, row] = x
    q = s["q_out"].double()
    q[:n] = spin(s["q"])
    return {"cache": cache, "q": q}


def _exact_evict(s, case):
    table, lens, mass = (s[k].cpu().numpy() for k in ("table", "lens", "mass"))
    n, cap, p = case["n_seqs"], case["cap"], case["tokens"]
    t_out, m_out, l_out = np.full_like(table, -1), np.zeros(mass.shape), lens.copy()
    ids, at, count = np.full((n, cap), -1, np.int32), np.full((n, cap), -1, np.int32), np.zeros(n, np.int32)
    for i in range(n):
        held = -(-int(lens[i]) // p)
        may = list(range(case["first"], max(case["first"], held - case["last"])))
        go = sorted(sorted(may, key=lambda j: (mass[i, j], j))[:min(max(held - case["budget"], 0), len(may), cap)])
        stay = sorted(set(range(held)) - set(go))
        t_out[i, :len(stay)], m_out[i, :len(stay)] = table[i, stay], mass[i, stay]
        ids[i, :len(go)], at[i, :len(go)] = table[i, go], go
        l_out[i] -= len(go) * p
        count[i] = len(go)
    return {"table": t_out, "mass": m_out, "lens": l_out, "ids": ids, "at": at, "count": count}
