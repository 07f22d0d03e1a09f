"""Attention of many rows with every token looked for by itself.  Bounds that follow from rounding are wider than one token's weight where
there are thousands; here each key is a vector of random signs, and a row asks for one of them: its score is 60, and others' are so much lower that the
row's result is that token's value and its log of the sum 60.  A token that is lost, taken twice or read from another's row shows at once."""
import math

import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import rows_reference as R

KIND = {"bf16": B.KV_BF16, "fp16": B.KV_FP16, "fp8": B.KV_FP8, "fp4": B.KV_FP4}
X = {"bf16": torch.bfloat16, "fp16": torch.float16}
SCORE = 60.0


def wrong(out, lse, value, x):
    """Which rows have not found their token.  A weight is off by half a step as it meets the value, and so is the result.  Others' scores are
    sums of as many random signs as there are dimensions, 64 and more, times 60 over that: one of 2^32 is above 48 or so, which has 2^-17 of the
    weight, and 2^15 of 30 have 2^-28; so 2^-10 of the row's largest value is room enough.  The log is off by those, and by (dim + 8) 2^-24 of 60."""
    off = (out.double() - value).abs()
    most = torch.finfo(x).eps * (1 + 2.0 ** -6) * value.abs() + 2.0 ** -10 * value.abs().amax(-1, keepdim=True)
    return ~(off <= most).all(-1) | ~((lse.double() - SCORE).abs() <= 2.0 ** -8)


class Probes:
    def __init__(self, new, lens, heads, group, dim, types=("bf16", "bf16"), p=16, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.x, self.types, self.heads, self.group, self.dim, self.p, self.device = X[types[0]], types, heads, group, dim, p, device
        self.new, self.lens = new, lens
        held = [-(-n // p) for n in lens]
        self.n_blocks = sum(held) + 1
        order = torch.randperm(self.n_blocks, generator=torch.Generator().manual_seed(seed)).int()
        self.table = torch.full((len(lens), max(max(held), 1)), -1, dtype=torch.int32)
        at = 0
        for s, h in enumerate(held):
            self.table[s, :h] = order[at:at + h]
            at += h
        fp4 = types[1] == "fp4"
        n = self.n_blocks * p
        keys = torch.randint(0, 2, (n, heads, dim), generator=g, device=device, dtype=torch.int8) * 2 - 1
        if fp4:
            codes = torch.randint(0, 16, (n, heads * dim), generator=g, device=device, dtype=torch.uint8)
            powers = torch.randint(124, 131, (n, heads * dim // 32), generator=g, device=device, dtype=torch.uint8)
            k = torch.where(keys.flatten(1) < 0, 10, 2).to(torch.uint8)      # 1 with its sign
            planes = [torch.cat([c[:, 0::2] | c[:, 1::2] << 4, e], 1) for c, e in ((k, torch.full_like(powers, 127)), (codes, powers))]
            numbers = R.NUMBERS.to(device)[(codes & 7).long()] * torch.where(codes >= 8, -1.0, 1.0).double()
            self.values = (numbers.unflatten(-1, (-1, 32)) * torch.exp2(powers.double() - 127)[..., None]).view(n, heads, dim)
        else:
            kind = torch.float8_e4m3fn if types[1] == "fp8" else self.x
            v = torch.randn((n, heads, dim), generator=g, device=device).to(kind)
            planes, self.values = [keys.to(kind).view(torch.uint8), v.view(torch.uint8)], v
        self.keys = keys
        self.cache = torch.stack(planes)[None].contiguous()
        self.shape = W.KVShape(1, heads, D.fp4_head_bytes(dim) if fp4 else dim, p, self.n_blocks, 1, 1 if types[1] in ("fp8", "fp4") else 2)
        # of every head of a row: its request, its place (a row's own token), its row and its head
        self.starts = torch.tensor([0] + list(new)).cumsum(0).int()
        self.n_rows = int(self.starts[-1])
        self.of = torch.cat([torch.full((m,), s) for s, m in enumerate(new)]).to(device)
        self.place = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, new)]).to(device)
        self.kv_head = torch.arange(heads * group, device=device) // group

    def cells(self, tokens):
        """tokens [row, head] -> rows of the cache"""
        page = self.table.to(self.device)[self.of[:, None], tokens // self.p]
        return page.long() * self.p + tokens % self.p

    def queries(self, tokens):
        return self.keys[self.cells(tokens), self.kv_head].to(self.x)

    def wanted(self, tokens):
        return self.values[self.cells(tokens), self.kv_head].double()

    def rounds(self, causal):
        """Tokens to ask for, [row, head] each time, until every request's tokens have all been asked for by some row; then each row's own
        token and the one before it."""
        heads = self.heads * self.group
        # (a KV head's tokens are asked for by its own heads of rows)
        sees = self.place - (self.place - torch.tensor(self.lens, device=self.device)[self.of] + torch.tensor(self.new, device=self.device)[self.of]) \
            if causal else torch.tensor(self.lens, device=self.device)[self.of] - 1
        sees = sees.clamp(min=0)                # the last token that all of the request's rows see
        row = torch.cat([torch.arange(m) for m in self.new]).to(self.device)
        flat = row[:, None] * self.group + torch.arange(heads, device=self.device)[None] % self.group
        many = max(-(-n // (m * self.group)) for n, m in zip(self.lens, self.new) if m)
        each = torch.tensor(self.new, device=self.device)[self.of] * self.group
        for i in range(many):
            yield (i * each[:, None] + flat) % (sees[:, None] + 1)
        yield (self.place if causal else sees)[:, None].expand(-1, heads)
        yield (self.place if causal else sees)[:, None].expand(-1, heads).sub(1).clamp(min=0)

    def check(self, causal=True, one=False):
        lens = torch.tensor(self.lens, dtype=torch.int32)
        dec = D.Decoder(B.make_config(self.shape), self.cache.data_ptr(), self.heads * self.group, max_seqs=len(self.lens), max_blocks=self.table.shape[1],
                        x_type=KIND[self.types[0]], kv_type=KIND[self.types[1]], weigh=False, max_rows=self.n_rows)
        table, lens, starts = self.table.cuda(), lens.cuda(), self.starts.cuda()
        scale = SCORE / self.dim
        out = torch.empty((self.n_rows, self.heads * self.group, self.dim), dtype=self.x, device="cuda")
        lse = torch.empty(out.shape[:2], device="cuda")

        def call(q):
            out.fill_(math.nan)
            lse.fill_(math.nan)
            if one:
                assert dec.kv_attend(0, q, table, lens, out, scale=scale, lse=lse) == B.KV_OK
            else:
                assert dec.kv_attend_rows(0, q, table, lens, out, starts=starts, causal=causal, scale=scale, lse=lse) == B.KV_OK

        bad = torch.zeros((), dtype=torch.int64, device="cuda")
        example = torch.full((3,), -1, dtype=torch.int64, device="cuda")
        for tokens in self.rounds(causal):
            call(self.queries(tokens))
            w = wrong(out, lse, self.wanted(tokens), self.x)
            bad += w.sum()
            at = w.flatten().long().argmax()
            example = torch.where(w.any() & (example[0] < 0), torch.stack([at // w.shape[1], at % w.shape[1], tokens.flatten()[at]]), example)
        assert bad.item() == 0, f"{bad.item()} tokens not found, for instance row, head, token {example.tolist()}"
        if causal:      # and nobody finds the token behind its own
            last = self.place + 1 < torch.tensor(self.lens, device="cuda")[self.of]
            if last.any():
                tokens = torch.where(last, self.place + 1, self.place)[:, None].expand(-1, out.shape[1])
                call(self.queries(tokens))
                assert (lse[last] < 50).all()


def short(v):
    return f"{len(v)} to {max(v)}" if isinstance(v, tuple) else str(v)


TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp8"), ("bf16", "fp4")]


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("new,lens,heads,group,dim,p", [
    ((5,), (20011,), 2, 4, 64, 16), ((1,), (4097,), 1, 8, 128, 5), ((3, 2, 0, 7), (20011, 517, 90, 4097), 2, 5, 64, 16),     # tiles of 32
    ((2,) * 70, (300,) * 30 + (5003,) + (90,) * 39, 2, 4, 64, 16),
    ((40,), (20011,), 2, 4, 64, 16), ((33, 60, 90), (4097, 60, 20011), 2, 5, 128, 24), ((300,), (4097,), 3, 1, 256, 16),       # of 128
    ((300,), (4097,), 64, 4, 64, 16), ((1100, 1030), (4097, 1030), 32, 1, 128, 7)], ids=short)                                   # of 256
def test_every_token_is_found(types, new, lens, heads, group, dim, p):
    Probes(new, lens, heads, group, dim, types, p, seed=len(lens) + dim).check()


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("new,lens,heads,group,dim", [((4, 2), (9001, 4097), 2, 4, 64), ((100, 40), (4097, 9001), 2, 4, 96), ((1100,), (1500,), 64, 1, 64)], ids=short)
def test_every_token_is_found_by_rows_that_see_all(types, new, lens, heads, group, dim):
    Probes(new, lens, heads, group, dim, types, seed=dim).check(causal=False)


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("new,lens", [((1024,) + (1,) * 60, (1024,) + tuple(4001 + 431 * i for i in range(60))),
                                      ((2048,) + (1,) * 255, (2048,) + tuple(500 + 7 * i for i in range(255)))], ids=["60 singles", "255 singles"])
def test_a_prompt_beside_many_single_rows(types, new, lens):
    """One call for a chunk of a prompt and other requests' next tokens, in tiles of 128 rows and of 32."""
    Probes(new, lens, 2, 4, 64, types, seed=5).check()


@pytest.mark.gpu
@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("lens,heads,group,dim", [((4097,), 2, 8, 64), ((300,) * 30 + (5003,) + (90,) * 39, 2, 4, 128), ((1500, 2047), 1, 20, 256)], ids=short)
def test_every_token_is_found_one_at_a_time(types, lens, heads, group, dim):
    Probes((1,) * len(lens), lens, heads, group, dim, types, seed=dim).check(one=True)


@pytest.mark.parametrize("fault", ["lost", "taken twice", "its neighbour's value", "its neighbour's key"])
def test_what_the_probes_see(fault):
    """Plain attention on the CPU, right and with one token's mistake."""
    n, dim = 4097, 64
    c = Probes((1,), (n,), 1, 1, dim, device="cpu", seed=3)
    cells = c.cells(torch.arange(n)[None])[0]
    k, v = c.keys[cells, 0].double(), c.values[cells, 0].double()
    tokens = torch.tensor([0, 1, 31, 32, 2047, 4096])
    q = k[tokens]

    def attend(mistake):
        out, lse = torch.empty((len(tokens), dim), dtype=torch.float64), torch.empty(len(tokens), dtype=torch.float64)
        for i, t in enumerate(tokens.tolist()):
            kk, vv, near = k.clone(), v.clone(), t - 1 if t else 1
            weight = torch.ones(n, dtype=torch.float64)
            if mistake == "lost":
                weight[t] = 0
            elif mistake == "taken twice":
                weight[t] = 2
            elif mistake == "its neighbour's value":
                vv[t] = v[near]
            elif mistake == "its neighbour's key":
                kk[t] = k[near]
            w = torch.exp(kk @ q[i] * (SCORE / dim)) * weight
            out[i], lse[i] = (w @ vv / w.sum()).to(c.x).double(), torch.log(w.sum())
        return wrong(out, lse, v[tokens], c.x)

    assert not attend("").any() and attend(fault).all()
