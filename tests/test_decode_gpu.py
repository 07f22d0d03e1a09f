"""The operators of a decode step (rotary writes into pages, paged attention of one new token,
eviction by weight) against plain implementations in 64 bits, at the sizes, masks and
layouts where they can go wrong."""
import math

import numpy as np
import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import decode_reference as R

pytestmark = pytest.mark.gpu

X = {"bf16": torch.bfloat16, "fp16": torch.float16}
KIND = {"bf16": B.KV_BF16, "fp16": B.KV_FP16, "fp8": B.KV_FP8}


class Case:
    """A cache with scattered pages, a decoder over it, and what its bytes stand for."""

    def __init__(self, heads=2, group=2, dim=64, p=16, lens=(5, 40), types=("bf16", "bf16"), layers=2, layer=1,
                 block_first=False, k_scale=1.0, v_scale=1.0, seed=0, extra_blocks=0, max_blocks=None, spread=1.0):
        self.g = torch.Generator().manual_seed(1000 + seed)
        self.rng = np.random.default_rng(seed)
        self.heads, self.group, self.dim, self.p, self.layer = heads, group, dim, p, layer
        self.x, self.types, self.scales = X[types[0]], types, (k_scale, v_scale)
        self.lens = torch.tensor(lens, dtype=torch.int32)
        held = [-(-max(0, n) // p) for n in lens]
        self.max_blocks = max(max(held), 1) + extra_blocks if max_blocks is None else max_blocks
        self.n_blocks = sum(min(h, self.max_blocks) for h in held) + 3
        order = iter(self.rng.permutation(self.n_blocks).tolist())
        self.table = torch.full((len(lens), self.max_blocks), -1, dtype=torch.int32)
        for s, h in enumerate(held):
            for j in range(min(h, self.max_blocks)):
                self.table[s, j] = next(order)
        shape = W.KVShape(layers, heads, dim, p, self.n_blocks, 1, 1 if types[1] == "fp8" else 2)
        self.block_first, self.layers = block_first, layers
        dims = (self.n_blocks, layers, 2, p, heads, dim) if block_first else (layers, 2, self.n_blocks, p, heads, dim)
        values = torch.randn(dims, generator=self.g) * spread
        if types[1] == "fp8":
            sc = torch.tensor([k_scale, v_scale]).view((1, 1, 2, 1, 1, 1) if block_first else (1, 2, 1, 1, 1, 1))
            self.cache = (values / sc).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        else:
            self.cache = values.to(self.x).cuda()
        self.cfg = B.make_config(shape, hbm_layout=1 if block_first else 0)
        self.dec = D.Decoder(self.cfg, self.cache.data_ptr(), heads * group, max_seqs=len(lens), max_blocks=self.max_blocks,
                             x_type=KIND[types[0]], kv_type=KIND[types[1]], k_scale=k_scale, v_scale=v_scale)

    def plane(self, which, cache=None):
        c = self.cache if cache is None else cache
        return c[:, self.layer, which] if self.block_first else c[self.layer, which]

    def values(self, which, cache=None):
        t = self.plane(which, cache).cpu()
        return t.view(torch.float8_e4m3fn).double() * self.scales[which] if self.types[1] == "fp8" else t.double()

    def queries(self, much=1.0):
        return (torch.randn((len(self.lens), self.heads * self.group, self.dim), generator=self.g) * much).to(self.x)

    def check_attend(self, q, scale=None, mass=True, lse=True, table=None, lens=None, **kw):
        """One call against the reference; returns what the call gave."""
        table, lens = self.table if table is None else table, self.lens if lens is None else lens
        ref = R.attend(q.double(), self.values(0), self.values(1), table, lens, scale or 1 / math.sqrt(self.dim), self.n_blocks)
        n = len(lens)
        qd, td, ld = q.cuda(), table.cuda(), lens.cuda()
        out = torch.full(q.shape, float("nan"), dtype=self.x, device="cuda")
        l_out = torch.full((n, q.shape[1]), float("nan"), device="cuda") if lse else None
        before = torch.rand((n, self.max_blocks), generator=self.g) if mass else None
        m_in = before.cuda() if mass else None
        m_out = torch.full_like(m_in, float("nan")) if mass else None
        rc = self.dec.kv_attend(self.layer, qd, td, ld, out, scale=scale, lse=l_out, mass=m_in, mass_out=m_out, **kw)
        assert rc == B.KV_OK, B.kv_strerror(rc)
        torch.cuda.synchronize()
        bound, lse_bound, mass_bound = R.attend_bounds(ref, lens, self.dim, self.x)
        off = (out.cpu().double() - ref["out"]).abs()
        assert not torch.isnan(off).any() and (off <= bound).all(), f"out off by {(off / bound).max():.2f} of the bound"
        if lse:
            got, empty = l_out.cpu().double(), torch.isinf(ref["lse"])
            assert torch.equal(torch.isinf(got) & (got < 0), empty)
            off = torch.where(empty, 0.0, (got - ref["lse"]).abs())
            assert (off <= lse_bound).all(), f"lse off by {(off / lse_bound).max():.2f} of the bound"
        if mass:
            off = (m_out.cpu().double() - before.double() - ref["mass"]).abs()
            bound = mass_bound + 2.0 ** -24 * (before.double() + ref["mass"])
            assert (off <= bound).all(), f"mass off by {(off / bound).max():.2f} of the bound"
            assert torch.equal(m_in.cpu(), before)
        return out, l_out, m_out


ALL_TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp8"), ("fp16", "fp8")]


@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
@pytest.mark.parametrize("heads,group,dim", [(2, 2, 64), (8, 4, 128), (1, 8, 128), (3, 3, 40), (4, 1, 256), (2, 16, 128), (1, 24, 96),
                                             (1, 40, 64), (5, 7, 80), (9, 2, 8), (2, 5, 192), (16, 1, 128), (4, 8, 32)])
def test_heads_and_dimensions(types, heads, group, dim):
    c = Case(heads, group, dim, lens=(1, 33, 100, 0, 64, 17, 130), types=types, k_scale=0.02 if types[1] == "fp8" else 1.0,
             v_scale=0.01 if types[1] == "fp8" else 1.0, seed=dim)
    c.check_attend(c.queries())


@pytest.mark.parametrize("p", [1, 2, 3, 4, 5, 7, 8, 12, 16, 20, 24, 32, 48, 100])
@pytest.mark.parametrize("block_first", [False, True])
def test_block_sizes_and_layouts(p, block_first):
    c = Case(2, 4, 64, p, lens=(1, 2, 31, 32, 33, 200, 0, 95, 64), block_first=block_first, layers=3, layer=2, seed=p)
    c.check_attend(c.queries())


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 256, 257, 1000, 4097, 20011])
@pytest.mark.parametrize("heads,group", [(1, 4), (8, 2)])
def test_lengths(n, heads, group):
    c = Case(heads, group, 64, lens=(n,), seed=n)
    c.check_attend(c.queries())


def test_many_requests_of_all_lengths():
    rng = np.random.default_rng(3)
    lens = np.concatenate([rng.integers(0, 3, 70), rng.integers(0, 300, 120), [0, 0, 0, 1500]])
    rng.shuffle(lens)
    c = Case(2, 3, 64, lens=tuple(int(n) for n in lens), seed=4, extra_blocks=2)
    c.check_attend(c.queries())


def test_only_empty_requests():
    c = Case(2, 2, 64, lens=(0, 0, -3), max_blocks=2)
    out, lse, _ = c.check_attend(c.queries())
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("p", [5, 16])
@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
def test_pages_that_are_not_there(p, types):
    """Ids below 0 and beyond the cache are skipped, wherever they stand; a request of nothing but such is empty."""
    c = Case(2, 2, 64, p, lens=(100, 90, 64, 16, 1), types=types, seed=7)
    t = c.table
    t[0, 0], t[0, 2], t[1, -1 - (c.max_blocks - -(-90 // p))] = -1, c.n_blocks, -5
    t[2, :] = 2 ** 31 - 1
    t[3, 0] = -2 ** 31
    if p == 5:
        t[3, :] = c.n_blocks + 1
    c.check_attend(c.queries())


@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
@pytest.mark.parametrize("p,dim", [(5, 40), (16, 128), (32, 96)])
def test_anything_behind_the_last_token(types, p, dim):
    """NaN and infinities in rows that no request has reached, in free blocks and in other heads change nothing."""
    c = Case(2, 2, dim, p, lens=(1, 13, 37, 0, p + 1), types=types, seed=8)
    q = c.queries()
    want = c.check_attend(q)
    bad = torch.ones((c.n_blocks, p), dtype=torch.bool)
    for s, n in enumerate(c.lens.tolist()):
        for t in range(n):
            bad[c.table[s, t // p], t % p] = False
    fill = [0x7F, 0xFF] if types[1] == "fp8" else [float("nan"), float("inf")]
    for which in (0, 1):
        c.plane(which).masked_fill_(bad.cuda()[:, :, None, None], fill[which])
    # and in every other plane
    for layer in range(c.layers):
        if layer != c.layer:
            (c.cache[:, layer] if c.block_first else c.cache[layer]).fill_(fill[0])
    again = c.check_attend(q)
    assert torch.equal(want[0], again[0]) and torch.equal(want[1], again[1])


def test_nan_of_one_head_stays_there():
    """A head whose dimensions do not fill a step of the products must not see its neighbour's NaN."""
    c = Case(3, 2, 40, lens=(50, 20), seed=9)
    q = c.queries()
    want, _, _ = c.check_attend(q)
    c.plane(0)[:, :, 1] = float("nan")
    out = torch.empty_like(want)
    assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out) == 0
    out = out.cpu()
    assert out[:, 2:4].isnan().all()
    assert torch.equal(out[:, :2], want.cpu()[:, :2]) and torch.equal(out[:, 4:], want.cpu()[:, 4:])


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp16")], ids="-".join)
@pytest.mark.parametrize("much", [0.0, 1e-3, 8.0, 60.0])
def test_flat_and_sharp_scores(types, much):
    c = Case(2, 4, 128, lens=(3000, 700), types=types, seed=11)
    c.check_attend(c.queries(much))


def test_scores_that_rise_along_the_request():
    """Every tile has a new largest score, by more than the slack; and the other way round."""
    c = Case(1, 2, 64, lens=(1024, 1024), seed=12)
    ramp = torch.linspace(-40, 40, 1024)
    for s, r in ((0, ramp), (1, ramp.flip(0))):
        for t in range(1024):
            c.plane(0)[c.table[s, t // 16], t % 16] = r[t].item()
    c.check_attend(torch.ones((2, 2, 64), dtype=torch.bfloat16))


def test_scores_of_minus_infinity_and_the_lowest_value():
    """Keys that give -inf weigh nothing beside others; the type's lowest value is a score like any."""
    c = Case(1, 2, 64, lens=(40, 40), seed=13)
    c.plane(0)[c.table[0, 0], 3, 0, 0] = float("-inf")
    c.plane(0)[c.table[1, 1], 2, 0, 0] = torch.finfo(torch.bfloat16).min
    q = c.queries().abs() + 1
    c_q = q.cuda()
    out, lse = torch.empty_like(c_q), torch.empty((2, 2), device="cuda")
    assert c.dec.kv_attend(c.layer, c_q, c.table.cuda(), c.lens.cuda(), out, lse=lse) == 0
    k = c.values(0)
    k[torch.isinf(k)] = -1e30
    ref = R.attend(q.double(), k, c.values(1), c.table, c.lens, 0.125, c.n_blocks)
    ref["size"] = ref["size"].clamp(max=40.0)       # of the scores that weigh anything
    bound, lse_bound, _ = R.attend_bounds(ref, c.lens, 64, torch.bfloat16)
    assert ((out.cpu().double() - ref["out"]).abs() <= bound).all()
    assert ((lse.cpu().double() - ref["lse"]).abs() <= lse_bound).all()


def test_equal_keys_average_the_values():
    """All weights equal, in a way that 16 bits cannot hold: out is the mean to half a step of the result (the rounded
    weights are divided by their own sum), and the masses are exact to 32 bits."""
    for types in (("bf16", "bf16"), ("fp16", "fp16")):
        c = Case(1, 2, 64, lens=(30000,), types=types, seed=14)
        c.plane(0).fill_(0.37)
        c.plane(1).fill_(1.5)
        out, lse, _ = c.check_attend(torch.full((1, 2, 64), 0.711, dtype=c.x))
        assert (out == 1.5).all()


def test_strided_queries_and_outputs():
    c = Case(2, 2, 64, lens=(50, 20, 3), seed=15)
    q = c.queries()
    want, _, _ = c.check_attend(q)
    wide = torch.zeros((3, 9, 64), dtype=c.x, device="cuda")
    wide[:, 2:6] = q.cuda()
    by_head = torch.zeros((4, 3, 72), dtype=c.x, device="cuda")     # [head, request, dim + padding]
    out = by_head.transpose(0, 1)[:, :, :64]
    table = torch.full((3, c.max_blocks + 5), -7, dtype=torch.int32, device="cuda")
    table[:, :c.max_blocks] = c.table.cuda()
    assert c.dec.kv_attend(c.layer, wide[:, 2:6], table[:, :c.max_blocks], c.lens.cuda(), out) == 0
    assert torch.equal(out, want) and (by_head[:, :, 64:] == 0).all()


def test_lengths_beyond_the_table_count_as_the_tables():
    c = Case(2, 2, 64, lens=(48, 48), seed=16)
    q = c.queries()
    want, _, _ = c.check_attend(q)
    out = torch.empty_like(want)
    lens = torch.tensor([48 + 7, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), lens, out) == 0
    assert torch.equal(out, want)


def test_fewer_requests_than_the_decoder_has_room_for_and_none():
    c = Case(2, 2, 64, lens=(48, 20, 100, 7), seed=17)
    q = c.queries()
    want, _, _ = c.check_attend(q)
    out = torch.full_like(want, 5.0)
    td, ld = c.table.cuda(), c.lens.cuda()
    for n in (0, 1, 3):
        assert c.dec.kv_attend(c.layer, q.cuda()[:n], td[:n], ld[:n], out[:n]) == 0
        # the split goes by the requests of the call: same result to the rounding of its parts
        assert torch.allclose(out[:n].float(), want[:n].float(), atol=0.05, rtol=0.02)
    assert (out[3:] == 5.0).all()


def test_the_same_bits_every_time_and_masses_in_place():
    c = Case(4, 4, 128, lens=(3000, 12, 800), seed=18)
    q, t, n = c.queries().cuda(), c.table.cuda(), c.lens.cuda()
    outs, masses = [], []
    for _ in range(6):
        out, mass = torch.empty_like(q), torch.ones((3, c.max_blocks), device="cuda")
        assert c.dec.kv_attend(c.layer, q, t, n, out, mass=mass) == 0
        outs.append(out), masses.append(mass)
    assert all(torch.equal(o, outs[0]) for o in outs) and all(torch.equal(m, masses[0]) for m in masses)
    alone = torch.empty_like(masses[0])
    assert c.dec.kv_attend(c.layer, q, t, n, outs[0], mass_out=alone) == 0
    assert torch.allclose(alone + 1, masses[0], atol=1e-5)
    assert torch.allclose(alone.sum(1), torch.full((3,), 16.0, device="cuda"), atol=1e-4)


def test_cells_beyond_32_bits():
    """A plane of more than 4 GiB: pages at both of its ends."""
    shape = W.KVShape(1, 8, 128, 16, 150000, 1)
    cache = torch.zeros(shape.cache_dims(), dtype=torch.bfloat16, device="cuda")
    dec = D.Decoder(B.make_config(shape), cache.data_ptr(), 8, max_seqs=1, max_blocks=4)
    ids = [149999, 0, 131073, 140001]
    g = torch.Generator().manual_seed(5)
    k = torch.randn((64, 8, 128), generator=g).to(torch.bfloat16).cuda()
    v = torch.randn((64, 8, 128), generator=g).to(torch.bfloat16).cuda()
    table, lens = torch.tensor([ids], dtype=torch.int32, device="cuda"), torch.tensor([64], dtype=torch.int32, device="cuda")
    assert dec.kv_put(0, k, v, table, lens, starts=torch.tensor([0, 64], dtype=torch.int32, device="cuda")) == 0
    assert torch.equal(cache[0, 0, ids].reshape(64, 8, 128), k) and torch.equal(cache[0, 1, ids].reshape(64, 8, 128), v)
    q = torch.randn((1, 8, 128), generator=g).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    assert dec.kv_attend(0, q, table, lens, out) == 0
    ref = R.attend(q.cpu().double(), cache[0, 0, ids].cpu().double(), cache[0, 1, ids].cpu().double(),
                   torch.arange(4)[None], lens.cpu(), 128 ** -0.5, 4)
    bound, _, _ = R.attend_bounds(ref, lens.cpu(), 128, torch.bfloat16)
    assert ((out.cpu().double() - ref["out"]).abs() <= bound).all()


# ---- new tokens --------------------------------------------------------------------------------

def check_put(c, news, rope=None, positions=None, with_q=True, behind=0, fused=False, in_place=False):
    """`news` new tokens per request, the last ones; every byte of the cache and of q is looked at."""
    rows = sum(news) + behind
    make = lambda h: torch.randn((rows, h, c.dim), generator=c.g).to(c.x)   # noqa: E731
    qh = c.heads * c.group
    if fused:
        qkv = make(qh + 2 * c.heads).cuda()
        q, k, v = qkv[:, :qh], qkv[:, qh:qh + c.heads], qkv[:, qh + c.heads:]
    else:
        q, k, v = make(qh).cuda(), make(c.heads).cuda(), make(c.heads).cuda()
    starts = np.concatenate([[0], np.cumsum(news)])
    each = None if all(n == 1 for n in news) and not behind else torch.tensor(starts, dtype=torch.int32, device="cuda")
    q_host, k_host, v_host = q.cpu(), k.cpu(), v.cpu()
    before = c.cache.clone()
    q_out = q if in_place else torch.full((rows, qh, c.dim), 7.0, dtype=c.x, device="cuda")
    rc = c.dec.kv_put(c.layer, k, v, c.table.cuda(), c.lens.cuda(), q=q if with_q else None, q_out=q_out if with_q else None,
                      starts=each, rope=rope, positions=None if positions is None else positions.cuda())
    assert rc == B.KV_OK, B.kv_strerror(rc)
    torch.cuda.synchronize()
    total = sum(news)
    place = [int(c.lens[s]) - n + i for s, n in enumerate(news) for i in range(n)]
    pos = torch.tensor(place)[None] if positions is None else positions[:, :total]
    turn = (lambda x: R.turned(x[:total], pos, rope.inv_freq.cpu(), rope.sections, 2 * rope.inv_freq.numel(), rope.interleaved)) \
        if rope else (lambda x: x[:total].double())
    # a turned value: two products and an addition in 32 bits of factors that are off by 2^-22, then rounded
    size = lambda x: x[:total].double().abs().amax(-1, keepdim=True)        # noqa: E731
    if with_q:
        want, u = turn(q_host), R.HALF_STEP[c.x]
        got = q_out.cpu().double()
        assert ((got[:total] - want).abs() <= u * want.abs() + 2.0 ** -20 * size(q_host) + 2.0 ** -24).all()
        rest = q_host[total:].double() if in_place else torch.full_like(got[total:], 7.0)
        assert torch.equal(got[total:], rest)
    expect = [c.plane(w, before).cpu().clone() for w in (0, 1)]
    seq = [s for s, n in enumerate(news) for _ in range(n)]
    for which, x in ((0, turn(k_host)), (1, v_host[:total].double())):
        got = c.plane(which).cpu()
        for i, (s, t) in enumerate(zip(seq, place)):
            if t < 0 or t >= c.max_blocks * c.p or not 0 <= int(c.table[s, t // c.p]) < c.n_blocks:
                continue
            cell = (int(c.table[s, t // c.p]), t % c.p)
            if c.types[1] == "fp8":
                scaled = x[i] / c.scales[which]
                want = torch.where(scaled.isnan(), scaled, scaled.clamp(-448, 448))
                have = got[cell].view(torch.float8_e4m3fn).double()
                slack = 2.0 ** -4 * want.abs() + 2.0 ** -10 + 2.0 ** -20 * (scaled.abs().max() if which == 0 else 0)
            else:
                want, have = x[i], got[cell].double()
                slack = (R.HALF_STEP[c.x] * want.abs() + 2.0 ** -20 * want.abs().max() + 2.0 ** -24) if rope and which == 0 else 0 * want
            assert ((have - want).abs() <= slack).all()
            expect[which][cell] = got[cell]
        # nothing else of the plane
        same = expect[which].view(torch.uint8) if c.types[1] == "fp8" else expect[which].view(torch.int16)
        assert torch.equal(got.view(same.dtype), same)
    # nor of any other plane
    untouched = c.cache.clone()
    for which in (0, 1):
        c.plane(which, untouched).copy_(c.plane(which, before))
    assert torch.equal(untouched.view(torch.uint8), before.view(torch.uint8))
    return q_out


def rope_of(rot, sections=None, interleaved=False, theta=10000.0):
    freq = (theta ** -(torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)).float().cuda()
    return D.Rope(freq, sections, interleaved)


@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
@pytest.mark.parametrize("dim,rot,sections,interleaved", [
    (64, 64, None, False), (128, 128, (16, 24, 24), False), (128, 64, (8, 24), True), (40, 40, None, False), (40, 24, (0, 5, 7), True),
    (256, 256, None, False), (80, 40, (20,), False), (8, 8, None, True), (96, 8, (1, 2, 1), False), (192, 192, (96,), True)])
def test_put_turns_and_stores(types, dim, rot, sections, interleaved):
    scales = dict(k_scale=0.02, v_scale=0.0125) if types[1] == "fp8" else {}
    c = Case(2, 3, dim, lens=(30, 1, 16, 77), types=types, seed=dim + rot, **scales)
    axes = len(sections) if sections else 1
    pos = torch.randint(0, 200000, (axes, 8 + 1 + 3 + 40), generator=c.g, dtype=torch.int32)
    check_put(c, (8, 1, 3, 40), rope_of(rot, sections, interleaved, 500000.0), pos)


@pytest.mark.parametrize("p", [1, 3, 5, 16, 32])
@pytest.mark.parametrize("block_first", [False, True])
def test_put_pages(p, block_first):
    c = Case(3, 2, 64, p, lens=(40, 7, 1, 100), block_first=block_first, layers=3, seed=p)
    check_put(c, (33, 7, 1, 50), rope_of(64), fused=True)


def test_put_one_each_without_starts_and_without_anything_to_turn():
    c = Case(8, 4, 128, lens=(40, 7, 1, 100), seed=1)
    check_put(c, (1, 1, 1, 1), rope_of(128))
    check_put(c, (1, 1, 1, 1), None)
    check_put(c, (1, 1, 1, 1), None, with_q=False)
    check_put(c, (1, 1, 1, 1), rope_of(128), with_q=False)
    check_put(c, (1, 1, 1, 1), rope_of(128), in_place=True)


def test_put_rows_behind_the_last_and_requests_without_rows():
    c = Case(2, 2, 64, lens=(40, 0, 7, 100, 5), seed=2)
    check_put(c, (4, 0, 7, 0, 2), rope_of(64), behind=9, fused=True)
    check_put(c, (0, 0, 0, 0, 0), rope_of(64), behind=3)


def test_put_skips_pages_that_are_not_there():
    """Missing pages and places outside the table stay out of the cache; q is turned all the same."""
    c = Case(2, 2, 64, 16, lens=(40, 33, 20), seed=3)
    c.table[0, 1] = -1
    c.table[1, 2] = c.n_blocks
    check_put(c, (20, 5, 20), rope_of(64))
    c.lens = torch.tensor([c.max_blocks * 16 + 2, 33, 3], dtype=torch.int32)    # two places beyond, two before the first
    check_put(c, (20, 5, 5), rope_of(64))


def test_put_far_positions_and_negative_ones():
    c = Case(1, 1, 128, lens=(64,), seed=4)
    pos = torch.cat([torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 1048575, -7]),
                     torch.randint(0, 2 ** 31 - 1, (59,), generator=c.g)]).to(torch.int32)[None]
    check_put(c, (64,), rope_of(128, theta=1e6), pos)


def test_put_eight_bits_at_the_borders():
    """Rounded to the nearest, ties to even, bounded to 448, NaN kept, small values and signs kept."""
    c = Case(1, 1, 64, lens=(1,), types=("fp16", "fp8"), seed=5)
    x = torch.tensor([448, 449, 464, 480, 1e4, -1e4, float("inf"), float("-inf"), float("nan"), 0.0, -0.0, 2.0 ** -9, 2.0 ** -10,
                      1.5 * 2.0 ** -9, 2.0 ** -11, 17, 18, 19, 21, 1.0625, 1.1875, -1.0625, 240, 248, 232] + [0.3] * 39).to(torch.float16)
    v = x.view(1, 1, 64).cuda()
    assert c.dec.kv_put(c.layer, v, v, c.table.cuda(), c.lens.cuda()) == 0
    want = torch.where(x.isnan(), x, x.clamp(-448, 448)).to(torch.float8_e4m3fn)
    for which in (0, 1):
        got = c.plane(which)[c.table[0, 0], 0, 0].cpu().view(torch.float8_e4m3fn)
        nan = want.float().isnan()
        assert torch.equal(got.float().isnan(), nan)
        assert torch.equal(got.view(torch.uint8)[~nan], want.view(torch.uint8)[~nan])


# ---- eviction ----------------------------------------------------------------------------------

def check_evict(table, lens, mass, p, budget, first, last, cap, in_place=False, dec=None):
    n, b = table.shape
    if dec is None:
        shape = W.KVShape(1, 1, 8, p, 4, 1)
        cache = torch.empty(shape.cache_dims(), dtype=torch.bfloat16, device="cuda")
        dec = D.Decoder(B.make_config(shape), cache.data_ptr(), 1, max_seqs=max(n, 1), max_blocks=b)
    want = R.evict(table, lens, mass, p, budget, first, last, cap)
    td, ld, md = table.cuda(), lens.cuda(), mass.cuda()
    to = {} if in_place else dict(table_out=torch.full_like(td, 99), lens_out=torch.full_like(ld, 99), mass_out=torch.full_like(md, 99))
    ids, at = (torch.full((n, cap), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    count = torch.full((n,), 99, dtype=torch.int32, device="cuda")
    rc = dec.kv_evict(td, ld, md, budget=budget, n_first=first, n_last=last, evicted_ids=ids, evicted_at=at, n_evicted=count, **to)
    assert rc == B.KV_OK, B.kv_strerror(rc)
    got = dict(table=to.get("table_out", td), lens=to.get("lens_out", ld), mass=to.get("mass_out", md), ids=ids, at=at, count=count)
    for name, x in got.items():
        a, w = x.cpu(), want[name]
        assert torch.equal(a.view(torch.int32), w.view(torch.int32)) if name != "mass" else \
            torch.equal(a.isnan(), w.isnan()) and torch.equal(a.nan_to_num(), w.nan_to_num()), name
    if not in_place:
        assert torch.equal(td.cpu(), table) and torch.equal(ld.cpu(), lens)
    return got


def evict_inputs(n, b, p, seed, lens=None, ties=False):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, b * p + 1, (n,), generator=g, dtype=torch.int32) if lens is None else torch.tensor(lens, dtype=torch.int32)
    mass = torch.randn((n, b), generator=g).exp()
    if ties:
        mass = torch.randint(0, 4, (n, b), generator=g).float()
    return torch.randperm(n * b, generator=g).to(torch.int32).view(n, b), lens, mass


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,b,p,budget,first,last,cap", [
    (1, 1, 16, 1, 0, 1, 1), (1, 2, 16, 1, 0, 1, 2), (7, 40, 16, 10, 1, 2, 40), (5, 100, 5, 0, 0, 1, 100), (3, 64, 16, 30, 4, 30, 64),
    (3, 64, 16, 2, 10, 10, 64), (4, 200, 16, 20, 1, 3, 7), (3, 1024, 16, 100, 1, 3, 1024), (2, 1025, 16, 1000, 0, 1, 1025),
    (2, 5000, 8, 777, 4, 32, 5000), (1, 70000, 1, 30000, 4, 100, 70000), (33, 17, 16, 5, 2, 2, 0), (2, 50, 16, 100, 1, 1, 50)])
def test_evict(n, b, p, budget, first, last, cap, in_place):
    for ties in (False, True):
        table, lens, mass = evict_inputs(n, b, p, seed=b + ties, ties=ties)
        lens[0] = b * p
        check_evict(table, lens, mass, p, budget, first, last, cap, in_place)


def test_evict_odd_weights_and_lengths():
    """NaN weighs most, -0 what 0 does; negative weights, infinities; lengths of none, of less and of more than the table."""
    table, lens, mass = evict_inputs(6, 300, 16, seed=2, lens=(4800, 0, -9, 2 ** 31 - 1, 17, 4799))
    g = torch.Generator().manual_seed(3)
    odd = torch.tensor([float("nan"), float("inf"), float("-inf"), 0.0, -0.0, -1.0, 1e-45, -1e-45, 3e38])
    mass = odd[torch.randint(0, 9, (6, 300), generator=g)]
    for budget in (0, 40, 150, 290):
        check_evict(table, lens, mass, 16, budget, 1, 2, 300)
    mass[:] = float("nan")
    check_evict(table, lens, mass, 16, 100, 1, 2, 300)
    mass[:] = 2.5
    check_evict(table, lens, mass, 16, 100, 3, 2, 300, in_place=True)


# ---- what is refused ---------------------------------------------------------------------------

def test_refusals_change_nothing():
    c = Case(2, 2, 64, lens=(40, 20), seed=6)
    q, t, n = c.queries().cuda(), c.table.cuda(), c.lens.cuda()
    out, k = torch.full_like(q, 3.0), torch.ones((2, 2, 64), dtype=c.x, device="cuda")
    before = c.cache.clone()
    att, put = c.dec.kv_attend, c.dec.kv_put
    EI, EU, E2 = B.KV_EINVAL, B.KV_EUNSUP, B.KV_E2BIG
    for layer in (-1, 2):
        assert att(layer, q, t, n, out) == EI and put(layer, k, k, t, n) == EI
    assert att(1, q.float(), t, n, out) == EI and att(1, q, t.long(), n, out) == EI and att(1, q, t, n.long(), out) == EI
    assert att(1, q.cpu(), t, n, out) == EI and att(1, q, t.cpu(), n, out) == EI
    assert att(1, q[:, :3], t, n, out) == EI and att(1, q, t[:, :1], n, out) == EI and att(1, q, t, n[:1], out) == EI
    assert att(1, q.transpose(1, 2), t, n, out) == EI and att(1, q, t, n, out[:, :, :32]) == EI and att(1, q[0], t, n, out) == EI
    assert att(1, q, t, n, out, scale=float("nan")) == EI and att(1, q, t, n, out, scale=float("inf")) == EI
    lse = torch.zeros((2, 4), device="cuda")
    assert att(1, q, t, n, out, lse=lse[:, :3]) == EI and att(1, q, t, n, out, lse=lse.double()) == EI
    assert att(1, q, t, n, out, mass=torch.zeros((2, c.max_blocks + 1), device="cuda")) == EI
    off = torch.zeros(2 * 4 * 64 + 8, dtype=c.x, device="cuda")
    assert att(1, off[4:516].view(2, 4, 64), t, n, out) == EU                       # 8 bytes behind a multiple of 16
    assert att(1, torch.zeros((2, 4, 68), dtype=c.x, device="cuda")[:, :, :64], t, n, out) == EU
    three = Case(2, 2, 64, lens=(40, 20, 1), max_blocks=c.max_blocks, seed=6)
    assert att(1, three.queries().cuda(), three.table.cuda(), three.lens.cuda(), torch.empty((3, 4, 64), dtype=c.x, device="cuda")) == E2
    assert put(1, k[:1], k, t, n) == EI and put(1, k, k[:, :1], t, n) == EI and put(1, k[:1], k[:1], t, n) == EI
    assert put(1, k, k, t, n, q=q) == EI and put(1, k, k, t, n, q=q, q_out=out[:1]) == EI
    assert put(1, k, k, t, n, starts=n) == EI
    rope = rope_of(64)
    assert put(1, k, k, t, n, rope=rope, positions=torch.zeros((2, 2), dtype=torch.int32, device="cuda")) == EI
    assert put(1, k, k, t, n, rope=rope, positions=torch.zeros((1, 3), dtype=torch.int32, device="cuda")) == EI
    assert put(1, k, k, t, n, positions=torch.zeros((1, 2), dtype=torch.int32, device="cuda")) == EI
    assert put(1, k, k, t, n, rope=rope_of(64, (16, 16))) == EI                     # two axes want positions
    assert put(1, k, k, t, n, rope=rope_of(128)) == EI
    assert put(1, k, k, t, n, rope=rope_of(12)) == EU
    ids, count, mass = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), \
        torch.zeros((2, c.max_blocks), device="cuda")
    ev = lambda **kw: c.dec.kv_evict(t, n, kw.pop("mass", mass), **{**dict(budget=1, n_first=0, n_last=1, evicted_ids=ids,  # noqa: E731
                                     evicted_at=ids.clone(), n_evicted=count), **kw})
    assert ev(budget=-1) == EI and ev(n_first=-1) == EI and ev(n_last=0) == EI and ev(mass=mass.double()) == EI
    assert ev(evicted_at=ids[:1]) == EI and ev(n_evicted=count.long()) == EI and ev(table_out=t[:1]) == EI
    torch.cuda.synchronize()
    assert torch.equal(c.cache, before) and (out == 3.0).all() and torch.equal(t.cpu(), c.table) and torch.equal(n.cpu(), c.lens)


def test_calls_that_raise_do_nothing():
    """What is no tensor, number or stream at all raises, before anything is launched."""
    c = Case(2, 2, 64, lens=(40, 20), seed=40)
    q, t, n = c.queries().cuda(), c.table.cuda(), c.lens.cuda()
    out, k, before = torch.full_like(q, 3.0), torch.ones((2, 2, 64), dtype=c.x, device="cuda"), c.cache.clone()
    mass = torch.zeros((2, c.max_blocks), device="cuda")
    ids, count = torch.full((2, 3), 9, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ev = dict(budget=1, n_first=0, n_last=1, evicted_ids=ids, evicted_at=ids.clone(), n_evicted=count)
    for stream in (torch.cuda.current_stream(), "0"):
        for call in (lambda s: c.dec.kv_attend(1, q, t, n, out, stream=s), lambda s: c.dec.kv_put(1, k, k, t, n, stream=s),
                     lambda s: c.dec.kv_evict(t, n, mass, stream=s, **ev)):
            with pytest.raises(TypeError):
                call(stream)
    with pytest.raises(TypeError):
        c.dec.kv_attend(1, q, t, n, out, scale="1")
    with pytest.raises(TypeError):
        c.dec.kv_attend(1.0, q, t, n, out)
    gone = D.Decoder(c.cfg, c.cache.data_ptr(), 4, max_seqs=2, max_blocks=c.max_blocks)
    assert gone.kv_decoder_destroy() == 0 and gone.kv_decoder_destroy() == 0
    with pytest.raises(ValueError):
        gone.kv_attend(1, q, t, n, out)
    # a gradient is asked for, and there is none
    asks = q.clone().requires_grad_()
    assert c.dec.kv_attend(1, asks, t, n, out) == B.KV_EINVAL
    torch.cuda.synchronize()
    assert (out == 3.0).all() and torch.equal(c.cache, before) and (ids == 9).all() and torch.equal(t.cpu(), c.table)
    with torch.no_grad():
        assert c.dec.kv_attend(1, asks, t, n, out) == 0


def test_decoders_that_cannot_be():
    def rc_of(shape, n_heads=4, ptr=None, elem=2, **kw):
        cache = torch.empty(2 * shape.n_layers * shape.n_hbm_blocks * shape.block_size * shape.n_kv_heads * shape.head_dim + 8,
                            dtype=torch.bfloat16, device="cuda")
        try:
            D.Decoder(B.make_config(shape), cache.data_ptr() if ptr is None else ptr(cache), n_heads,
                      **{**dict(max_seqs=2, max_blocks=2), **kw})
        except B.KVError as e:
            return e.code
        return 0
    sh = lambda dim=64, heads=2, elem=2: W.KVShape(1, heads, dim, 16, 4, 1, elem)   # noqa: E731
    assert rc_of(sh()) == 0
    assert rc_of(sh(), n_heads=3) == B.KV_EINVAL and rc_of(sh(), n_heads=0) == B.KV_EINVAL
    assert rc_of(sh(), max_seqs=0) == B.KV_EINVAL and rc_of(sh(), max_blocks=0) == B.KV_EINVAL
    assert rc_of(sh(), x_type=B.KV_BF16, kv_type=B.KV_FP16) == B.KV_EINVAL
    assert rc_of(sh(), kv_type=B.KV_FP8) == B.KV_EINVAL and rc_of(sh(elem=1)) == B.KV_EINVAL
    assert rc_of(sh(), k_scale=2.0) == B.KV_EINVAL
    for bad in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert rc_of(sh(elem=1), kv_type=B.KV_FP8, v_scale=bad) == B.KV_EINVAL
    assert rc_of(sh(dim=264)) == B.KV_EUNSUP and rc_of(sh(dim=60)) == B.KV_EUNSUP and rc_of(sh(heads=1), n_heads=1025) == B.KV_EUNSUP
    assert rc_of(sh(), ptr=lambda t: t.data_ptr() + 2) == B.KV_EUNSUP
    assert rc_of(sh(), ptr=lambda t: torch.empty(1 << 16, dtype=torch.uint8).data_ptr() // 16 * 16) == B.KV_EINVAL
    assert rc_of(W.KVShape(1, 2, 64, 16, 1 << 22, 1), ptr=lambda t: torch.empty(16, device="cuda").data_ptr()) == B.KV_EINVAL


# ---- together ----------------------------------------------------------------------------------

def test_decode_loop_recorded_and_replayed():
    """put, attend over two layers with weights, evict, in one graph: replayed as the requests grow, beside eager work,
    each replay against the same step run eagerly on a second copy of everything."""
    heads, group, dim, p, n, layers = 2, 4, 64, 16, 5, 2
    budget, max_blocks, n_blocks = 6, 9, 64
    g = torch.Generator().manual_seed(21)
    shape = W.KVShape(layers, heads, dim, p, n_blocks, 1)
    rope = rope_of(dim)

    class Side:
        def __init__(self):
            self.cache = torch.zeros(shape.cache_dims(), dtype=torch.bfloat16, device="cuda")
            self.dec = D.Decoder(B.make_config(shape), self.cache.data_ptr(), heads * group, max_seqs=n, max_blocks=max_blocks)
            z = lambda *d, t=torch.bfloat16: torch.zeros(d, dtype=t, device="cuda")     # noqa: E731
            self.qkv = z(layers, n, heads * (group + 2), dim)
            self.out = z(layers, n, heads * group, dim)
            self.table = torch.full((n, max_blocks), -1, dtype=torch.int32, device="cuda")
            self.lens, self.count, self.pos = z(n, t=torch.int32), z(n, t=torch.int32), z(1, n, t=torch.int32)
            self.mass = z(n, max_blocks, t=torch.float32)
            self.ids, self.at = z(n, 4, t=torch.int32), z(n, 4, t=torch.int32)

        def step(self):
            qh = heads * group
            for layer in range(layers):
                x = self.qkv[layer]
                q = x[:, :qh]
                assert self.dec.kv_put(layer, x[:, qh:qh + heads], x[:, qh + heads:], self.table, self.lens, q=q, q_out=q,
                                       rope=rope, positions=self.pos) == 0
                assert self.dec.kv_attend(layer, q, self.table, self.lens, self.out[layer], mass=self.mass) == 0
            assert self.dec.kv_evict(self.table, self.lens, self.mass, budget=budget, n_first=1, n_last=2, evicted_ids=self.ids,
                                     evicted_at=self.at, n_evicted=self.count) == 0

    eager, graphed = Side(), Side()
    graphed.step()                          # once outside any recording
    for s in (eager, graphed):
        s.mass.zero_(), s.cache.zero_()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        graphed.step()
    free = [list(range(n_blocks)) for _ in range(1)][0]
    grown = torch.zeros(n, dtype=torch.int64)
    seen = 0
    for it in range(150):
        qkv = torch.randn((layers, n, heads * (group + 2), dim), generator=g).to(torch.bfloat16)
        lens, table = eager.lens.cpu(), eager.table.cpu()
        for r in range(n):
            if (it + r) % 3 == 0 and r:     # not every request runs in every step, but its row of q does
                pass
            if int(lens[r]) % p == 0:
                table[r, int(lens[r]) // p] = free.pop(0)
            lens[r] += 1
            grown[r] += 1
        for s in (eager, graphed):
            s.qkv.copy_(qkv), s.lens.copy_(lens), s.table.copy_(table), s.pos.copy_((grown - 1)[None].to(torch.int32))
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("out", "cache", "table", "lens", "mass", "ids", "at", "count"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), f"{name} in step {it}"
        k = int(eager.count.sum())
        seen += k
        free += [int(i) for row, m in zip(eager.ids.cpu(), eager.count.cpu()) for i in row[:int(m)]]
        junk = torch.randn(1 << 16, device="cuda").sum()    # the program's own work between replays
        assert torch.isfinite(junk)
    assert seen == n * (10 - budget), seen       # 150 tokens are 10 blocks


def test_attend_beside_rotation_and_eviction_through_the_table():
    """The block table's own blocks: prompts are put, attended to, the lightest blocks leave through kv_evict and
    kv_table_drop, a request rotates out and in, and attends to the same as before."""
    shape = W.KVShape(2, 2, 64, 16, n_hbm_blocks=64, n_host_slots=64)
    cache = torch.zeros(shape.cache_dims(), dtype=torch.bfloat16, device="cuda")
    eng = B.Engine(B.make_config(shape), cache.data_ptr())
    tab = B.Table(eng, 4)
    dec = D.Decoder(eng.cfg, cache.data_ptr(), 4, max_seqs=2, max_blocks=16)
    g = torch.Generator().manual_seed(22)
    lengths = (200, 90)

    def tables(reqs):
        t, n = torch.full((len(reqs), 16), -1, dtype=torch.int32), torch.zeros(len(reqs), dtype=torch.int32)
        for i, r in enumerate(reqs):
            b = tab.kv_table_blocks(r)
            t[i, :len(b["ids"])], n[i] = torch.tensor(b["ids"], dtype=torch.int32), b["len"]
        return t.cuda(), n.cuda()

    for r, n in enumerate(lengths):
        assert tab.kv_table_append(r, n)[0] == 0
    t, n = tables((0, 1))
    rows = sum(lengths)
    kv = torch.randn((2, 2, rows, 2, 64), generator=g).to(torch.bfloat16).cuda()
    starts = torch.tensor([0, 200, 290], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 4, 64), generator=g).to(torch.bfloat16).cuda() * 2
    mass, out = torch.zeros((2, 16), device="cuda"), torch.empty((2, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
    for layer in range(2):
        assert dec.kv_put(layer, kv[layer, 0], kv[layer, 1], t, n, starts=starts, rope=rope_of(64)) == 0
        assert dec.kv_attend(layer, q, t, n, out[layer], mass=mass) == 0
    ids, at = (torch.zeros((2, 16), dtype=torch.int32, device="cuda") for _ in range(2))
    count = torch.zeros(2, dtype=torch.int32, device="cuda")
    heavy = mass.clone()
    assert dec.kv_evict(t, n, mass, budget=8, n_first=1, n_last=1, evicted_ids=ids, evicted_at=at, n_evicted=count) == 0
    assert count.tolist() == [13 - 8, 0]
    free = tab.kv_table_get_counts()["free_hbm_blocks"]
    for r in range(2):
        assert tab.kv_table_drop(r, at[r, :int(count[r])].cpu().numpy()) == 0
    assert tab.kv_table_get_counts()["free_hbm_blocks"] == free + 5
    t2, n2 = tables((0, 1))
    assert torch.equal(t2, t) and torch.equal(n2, n) and n.tolist() == [200 - 80, 90]
    gone = at[0, :5].long()
    assert heavy[0, gone].max() <= torch.cat([heavy[0, 1:12][~torch.isin(torch.arange(1, 12, device="cuda"), gone)]]).min()
    kept = torch.empty_like(out)
    for layer in range(2):
        assert dec.kv_attend(layer, q, t, n, kept[layer]) == 0
    torch.cuda.synchronize()
    # out to DRAM and back, into whichever blocks are free then
    assert tab.kv_table_rotate([0], []) == 0 and eng.kv_wait() == 0
    t3, n3 = tables((0, 1))
    assert (t3[0] == -1).all()
    away = torch.empty_like(q)
    assert dec.kv_attend(0, q, t3, n3, away) == 0
    assert (away[0] == 0).all()                      # what is in DRAM is not attended to
    assert tab.kv_table_append(2, 100)[0] == 0
    assert tab.kv_table_rotate([], [0]) == 0
    stream = torch.cuda.current_stream()
    assert eng.kv_stream_wait_layer(stream.cuda_stream, 1) == 0
    t4, n4 = tables((0, 1))
    assert not torch.equal(t4[0], t[0])
    back = torch.empty_like(out)
    for layer in range(2):
        assert dec.kv_attend(layer, q, t4, n4, back[layer]) == 0
    torch.cuda.synchronize()
    assert torch.equal(back, kept)
    assert eng.kv_wait() == 0
    tab.kv_table_destroy(), eng.kv_destroy()


def test_decode_command_runs_on_a_small_cache():
    """The command's own checks (recorded step equals eager, tables close up alike, blocks given back), then its rows."""
    from paper_2601_20309_amd import experiments as X
    got = X.decode("small8b", n_heads=32, n_run=6, n_rotate=2, rotate_tokens=160, budget=6, steps=3, longest=300)
    assert got["finite"] and got["evicted"] > 0 and len(got["rows"]) == 4 and got["rotated"]["gbs"] > 0
    assert got["rows"][3]["gib"] < got["rows"][0]["gib"]


@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
@pytest.mark.parametrize("n,longest,heads,group,dim,p", [
    (300, 192, 8, 2, 128, 16), (40, 64, 8, 4, 64, 16), (3, 600, 4, 4, 128, 16), (5, 300, 2, 3, 40, 5), (2, 256, 8, 4, 256, 16),
    (70, 130, 3, 3, 96, 16), (1, 33, 16, 2, 128, 8), (9, 1200, 2, 4, 64, 16)])
def test_short_tables_without_weights(n, longest, heads, group, dim, p, types):
    """A range per request with as many waves each as there is room for, one launch: lengths 0 to the longest."""
    lens = [longest] + np.random.default_rng(n).integers(0, longest + 1, n - 1).tolist()
    if n > 2:
        lens[1] = 0
    c = Case(heads, group, dim, p, lens=lens, types=types, seed=n, k_scale=0.02 if types[1] == "fp8" else 1.0)
    c.check_attend(c.queries(), mass=False)
    c.check_attend(c.queries(), mass=False, lse=False)


@pytest.mark.parametrize("p,heads,group,n,longest", [(5, 1, 8, 45, 8000), (5, 1, 4, 9, 700), (16, 1, 24, 3, 5000), (7, 2, 3, 40, 11000), (3, 1, 30, 5, 90)])
def test_weights_of_many_blocks(p, heads, group, n, longest):
    """Few and many numbers a block, few and many blocks: long tables of which requests fill little, but one."""
    lens = [longest // 8] + np.random.default_rng(p).integers(0, 400, n - 1).tolist()
    c = Case(heads, group, 40, p, lens=lens, max_blocks=-(-longest // p), seed=p + n)
    c.check_attend(c.queries())


def test_pages_that_several_entries_name():
    """A prefix that requests share, and one page twice in a row of the table: read as often as it is named."""
    c = Case(2, 4, 128, lens=(90, 75, 64), seed=41)
    table = c.table.clone()
    table[1, :3] = table[0, :3]
    table[2, 1] = table[2, 3] = table[2, 0]
    c.check_attend(c.queries(), table=table)


def test_put_of_broadcast_rows_and_positions():
    """One row of k, v and q for all tokens, and the same positions along every axis."""
    c = Case(2, 2, 64, lens=(20, 33, 5), seed=42)
    other = Case(2, 2, 64, lens=(20, 33, 5), seed=42)
    rope = rope_of(64, (16, 8, 8))
    one = [torch.randn((1, h, 64), generator=c.g).to(c.x).cuda() for h in (2, 2, 4)]
    k, v, q = (x.expand(3, -1, -1) for x in one)
    pos = torch.tensor([[7, 70000, 3]], dtype=torch.int32, device="cuda")
    outs = [torch.empty((3, 4, 64), dtype=c.x, device="cuda") for _ in range(2)]
    t, n = c.table.cuda(), c.lens.cuda()
    assert c.dec.kv_put(1, k, v, t, n, q=q, q_out=outs[0], rope=rope, positions=pos.expand(3, 3)) == 0
    assert other.dec.kv_put(1, k.contiguous(), v.contiguous(), t, n, q=q.contiguous(), q_out=outs[1], rope=rope,
                            positions=pos.expand(3, 3).contiguous()) == 0
    assert torch.equal(outs[0], outs[1]) and torch.equal(c.cache, other.cache)
    assert c.dec.kv_put(1, k, v, t, n, q=q, q_out=outs[0][:1].expand(3, 4, 64)) == B.KV_EINVAL


def test_two_recorded_calls_share_a_decoder():
    """Graphs of one decoder, replayed in turn on one stream, between eager calls through it."""
    c = Case(4, 4, 128, lens=(3000, 300, 17, 0), seed=43)
    t, n = c.table.cuda(), c.lens.cuda()
    few = torch.tensor([100, 2990, 0, 64], dtype=torch.int32).clamp(max=c.max_blocks * 16).cuda()
    q = [c.queries().cuda() for _ in range(2)]
    outs, masses = [torch.empty_like(x) for x in q], [torch.zeros((4, c.max_blocks), device="cuda") for _ in q]
    call = lambda i, out, mass: c.dec.kv_attend(i, q[i], t, (n, few)[i], out, mass_out=mass)    # noqa: E731
    want = []
    for i in range(2):
        o, m = torch.empty_like(q[i]), torch.zeros_like(masses[i])
        assert call(i, o, m) == 0
        want.append((o, m))
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            assert call(i, outs[i], masses[i]) == 0
        graphs.append(g)
    for turn in range(5):
        for i in (0, 1, 1, 0)[turn % 2:]:
            outs[i].fill_(float("nan"))
            masses[i].fill_(float("nan"))
            graphs[i].replay()
            o, m = torch.empty_like(q[1 - i]), torch.empty_like(masses[i])
            assert call(1 - i, o, m) == 0
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i][0]) and torch.equal(masses[i], want[i][1])
            assert torch.equal(o, want[1 - i][0]) and torch.equal(m, want[1 - i][1])


def test_evict_with_many_of_one_weight_and_close_ones():
    """Rows on both sides of where entries are compared instead of counted: many that begin alike, few, all equal."""
    for b in (300, 512, 513, 2048, 2049, 4096, 4097):
        table, lens, mass = evict_inputs(6, b, 16, seed=b, lens=(b * 16,) * 6)
        close = torch.rand((b,), generator=torch.Generator().manual_seed(b))
        mass[0] = 1.0 + close * 2.0 ** -12                  # all in one first digit
        mass[1] = 0.25
        mass[2] = torch.where(close < 0.5, 1.0, 1.0 + 2.0 ** -23)
        mass[3] = torch.where(close < 0.02, 1.0, 4.0 + close)
        mass[4] = close * 1e-38
        for budget in (1, b // 3, b - 3):
            check_evict(table, lens, mass, 16, budget, 1, 1, b)


def test_q_is_its_own_output_and_broadcast_queries():
    c = Case(4, 3, 128, lens=(700, 33, 0, 5), seed=31)
    q = c.queries()
    want, _, _ = c.check_attend(q, mass=False, lse=False)      # the same call: with weights the split is another
    mine = q.cuda()
    assert c.dec.kv_attend(c.layer, mine, c.table.cuda(), c.lens.cuda(), mine) == 0
    assert torch.equal(mine, want)
    one = q[:1, :1].cuda().expand(4, 12, 128)            # one query for all requests and heads
    same = one.contiguous()
    a, b = torch.empty_like(same), torch.empty_like(same)
    for x, o in ((one, a), (same, b)):
        assert c.dec.kv_attend(c.layer, x, c.table.cuda(), c.lens.cuda(), o) == 0
    assert torch.equal(a, b)
    assert c.dec.kv_attend(c.layer, same, c.table.cuda(), c.lens.cuda(), a[:1].expand(4, 12, 128)) == B.KV_EINVAL


def test_scores_near_the_lowest_float():
    """All scores of a row far below zero: the softmax is that of their differences."""
    c = Case(1, 1, 64, lens=(70,), seed=32, types=("bf16", "bf16"))
    c.plane(0).fill_(-1.0)
    q = torch.full((1, 1, 64), 3e36, dtype=torch.bfloat16)
    out = torch.empty((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out, scale=1.0) == 0
    v = c.values(1)
    mean = torch.stack([v[c.table[0, t // 16], t % 16, 0] for t in range(70)]).mean(0)
    size = torch.stack([v[c.table[0, t // 16], t % 16, 0] for t in range(70)]).abs().mean(0)
    assert ((out.cpu()[0, 0].double() - mean).abs() <= 2 ** -8 * (mean.abs() + 2 * size)).all()


def test_without_memory_for_weights():
    c = Case(2, 2, 64, lens=(50, 20), seed=33)
    light = D.Decoder(c.cfg, c.cache.data_ptr(), 4, max_seqs=2, max_blocks=c.max_blocks, weigh=False)
    q = c.queries()
    want, _, _ = c.check_attend(q)
    out, mass = torch.empty_like(want), torch.zeros((2, c.max_blocks), device="cuda")
    assert light.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out, mass=mass) == B.KV_EUNSUP
    assert light.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out) == 0
    assert torch.equal(out, want)


def test_two_decoders_on_two_streams():
    """Steps that overlap in time, each with its own decoder over one cache."""
    c = Case(4, 4, 128, lens=(5000, 300, 17), seed=30)
    other = D.Decoder(c.cfg, c.cache.data_ptr(), 16, max_seqs=3, max_blocks=c.max_blocks)
    q, t, n = [c.queries().cuda() for _ in range(2)], c.table.cuda(), c.lens.cuda()
    want = []
    for i in range(2):
        o = torch.empty_like(q[i])
        assert c.dec.kv_attend(c.layer, q[i], t, n, o) == 0
        want.append(o)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i, dec in enumerate((c.dec, other)):
            o = torch.empty_like(q[i])
            assert dec.kv_attend(c.layer, q[i], t, n, o, stream=streams[i].cuda_stream) == 0
            outs[i].append(o)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])
