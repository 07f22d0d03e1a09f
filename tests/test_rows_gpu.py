"""Attention of many rows over the paged cache against plain 64-bit arithmetic, at the sizes, masks and layouts where it can
go wrong."""
import math

import numpy as np
import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import rows_reference as R

pytestmark = pytest.mark.gpu

X = {"bf16": torch.bfloat16, "fp16": torch.float16}
KIND = {"bf16": B.KV_BF16, "fp16": B.KV_FP16, "fp8": B.KV_FP8, "fp4": B.KV_FP4}
ALL_TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp8"), ("fp16", "fp8"), ("bf16", "fp4"), ("fp16", "fp4")]


class Case:
    """A cache with scattered pages, requests with `new` rows each over `lens` tokens, and a decoder."""

    def __init__(self, new, lens, heads=2, group=2, dim=64, p=16, types=("bf16", "bf16"), layers=2, layer=1, block_first=False,
                 k_scale=1.0, v_scale=1.0, seed=0, max_blocks=None, behind=0, spread=1.0):
        self.g = torch.Generator().manual_seed(500 + seed)
        rng = np.random.default_rng(seed)
        self.heads, self.group, self.dim, self.p, self.layer, self.layers = heads, group, dim, p, layer, layers
        self.x, self.types, self.scales, self.block_first = X[types[0]], types, (k_scale, v_scale), block_first
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
        self.n_rows = int(self.starts[-1]) + behind
        held = [-(-max(0, n) // p) for n in lens]
        self.max_blocks = max(max(held), 1) if max_blocks is None else max_blocks
        self.n_blocks = sum(min(h, self.max_blocks) for h in held) + 3
        order = iter(rng.permutation(self.n_blocks).tolist())
        self.table = torch.full((len(lens), self.max_blocks), -1, dtype=torch.int32)
        for s, h in enumerate(held):
            for j in range(min(h, self.max_blocks)):
                self.table[s, j] = next(order)
        fp4 = types[1] == "fp4"
        shape = W.KVShape(layers, heads, D.fp4_head_bytes(dim) if fp4 else dim, p, self.n_blocks, 1, 1 if types[1] in ("fp8", "fp4") else 2)
        dims = (self.n_blocks, layers, 2, p, heads, dim) if block_first else (layers, 2, self.n_blocks, p, heads, dim)
        values = torch.randn(dims, generator=self.g) * spread
        if types[1] == "fp8":
            sc = torch.tensor([k_scale, v_scale]).view((1, 1, 2, 1, 1, 1) if block_first else (1, 2, 1, 1, 1, 1))
            self.host = (values / sc).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        elif fp4:
            self.host = R.fp4_rows(values, self.x)
        else:
            self.host = values.to(self.x)
        self.cache = self.host.cuda()
        self.cfg = B.make_config(shape, hbm_layout=1 if block_first else 0)
        self.dec = D.Decoder(self.cfg, self.cache.data_ptr(), heads * group, max_seqs=len(lens), max_blocks=self.max_blocks,
                             x_type=KIND[types[0]], kv_type=KIND[types[1]], k_scale=k_scale, v_scale=v_scale, weigh=False,
                             max_rows=max(self.n_rows, 1))

    def plane(self, which, cache=None):
        c = self.cache if cache is None else cache
        return c[:, self.layer, which] if self.block_first else c[self.layer, which]

    def values(self, which):
        t = self.plane(which).cpu()
        if self.types[1] == "fp4":
            return R.fp4_values(t, self.heads, self.dim)
        return t.view(torch.float8_e4m3fn).double() * self.scales[which] if self.types[1] == "fp8" else t.double()

    def queries(self, much=1.0):
        return (torch.randn((self.n_rows, self.heads * self.group, self.dim), generator=self.g) * much).to(self.x)

    def check(self, q=None, causal=True, scale=None, table=None, lens=None, starts=None, lse=True, **kw):
        q = self.queries() if q is None else q
        table, lens = self.table if table is None else table, self.lens if lens is None else lens
        starts = self.starts if starts is None else starts
        ref = R.rows(q, self.values(0), self.values(1), table, lens, starts, 1 / math.sqrt(self.dim) if scale is None else scale, causal,
                     self.n_blocks)
        mark = 7.0
        out = torch.full(q.shape, mark, dtype=self.x, device="cuda")
        l_out = torch.full(q.shape[:2], mark, device="cuda") if lse else None
        rc = self.dec.kv_attend_rows(self.layer, q.cuda(), table.cuda(), lens.cuda(), out, starts=starts.cuda(), causal=causal, scale=scale,
                                     lse=l_out, **kw)
        assert rc == B.KV_OK, B.kv_strerror(rc)
        torch.cuda.synchronize()
        self.compare(out, l_out, ref, mark)
        return out, l_out

    def compare(self, out, l_out, ref, mark=None):
        bound, lse_bound = R.rows_bounds(ref, self.dim, self.x)
        nobody = torch.isnan(ref["lse"][:, 0]) & torch.isnan(ref["size"][:, 0])
        got = out.cpu().double()
        if mark is not None:
            assert (got[nobody] == mark).all(), "rows of nobody were written"
        got, want, bound = got[~nobody], ref["out"][~nobody], bound[~nobody]
        same = (got == want) | (got.isnan() & want.isnan())
        off = (got - want).abs()
        assert (same | (off <= bound)).all(), f"out off by {(off / bound)[~same].max():.2f} of the bound"
        if l_out is not None:
            got = l_out.cpu().double()
            if mark is not None:
                assert (got[nobody] == mark).all()
            got, want, bound = got[~nobody], ref["lse"][~nobody], lse_bound[~nobody]
            same = (got == want) | (got.isnan() & want.isnan())
            off = (got - want).abs()
            assert (same | (off <= bound)).all(), f"lse off by {(off / bound)[~same].max():.2f} of the bound"


@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
@pytest.mark.parametrize("heads,group,dim", [(2, 2, 64), (8, 4, 128), (1, 8, 128), (3, 3, 96), (4, 1, 256), (1, 40, 64), (2, 5, 192), (2, 3, 32),
                                             (3, 2, 160), (5, 7, 224)])
def test_heads_and_dimensions(types, heads, group, dim):
    c = Case((1, 33, 100, 0, 64, 17, 3), (1, 33, 130, 5, 64, 90, 0), heads, group, dim, types=types, k_scale=0.02 if types[1] == "fp8" else 1.0,
             v_scale=0.01 if types[1] == "fp8" else 1.0, seed=dim, behind=5)
    c.check()
    c.check(causal=False)


@pytest.mark.parametrize("types", ALL_TYPES[:4], ids="-".join)
@pytest.mark.parametrize("heads,group,dim", [(3, 3, 40), (5, 7, 80), (9, 2, 8), (2, 2, 104), (1, 4, 200)])
def test_dimensions_that_are_no_multiple_of_32(types, heads, group, dim):
    c = Case((5, 70, 1), (100, 70, 33), heads, group, dim, p=5, types=types, seed=dim, k_scale=0.02 if types[1] == "fp8" else 1.0)
    c.plane(0)[:] = c.plane(0)          # (what lies behind a head's dimensions are the next one's)
    c.check()
    c.check(causal=False)


@pytest.mark.parametrize("p", [1, 2, 3, 5, 7, 8, 12, 16, 20, 24, 32, 48, 100])
@pytest.mark.parametrize("block_first", [False, True])
@pytest.mark.parametrize("kv", ["bf16", "fp4"])
def test_block_sizes_and_layouts(p, block_first, kv):
    c = Case((1, 2, 31, 32, 33, 20, 0, 95), (1, 2, 31, 40, 333, 200, 0, 95), 1, 4, 64, p, types=("bf16", kv), block_first=block_first, layers=3,
             layer=2, seed=p)
    c.check()


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000, 4097, 20011])
@pytest.mark.parametrize("new", [1, 2, 16, 33])
def test_lengths(n, new):
    c = Case((new,), (n,), 1, 4, 64, seed=n)
    c.check()
    c.check(causal=False)


@pytest.mark.parametrize("new", [127, 128, 129, 255, 257, 640])
def test_many_rows(new):
    c = Case((new, 1, new // 2), (new + 100, 1, new // 2), 2, 1, 128, seed=new)
    c.check()
    c.check(causal=False)


def test_more_rows_than_tokens():
    """Rows before a request's first token see nothing."""
    c = Case((40, 200, 7), (30, 3, 0), 2, 2, 64, seed=3)
    out, lse = c.check()
    assert (out[:10] == 0).all() and torch.isinf(lse[:10]).all() and not torch.isinf(lse[10:40]).any()


def test_many_requests():
    rng = np.random.default_rng(4)
    new = rng.integers(0, 4, 300)
    new[rng.integers(0, 300, 100)] = 0
    lens = rng.integers(0, 90, 300)
    lens[17], new[17] = 900, 50
    Case(new.tolist(), lens.tolist(), 1, 2, 64, p=8, seed=8).check()


def test_one_row_each_without_starts():
    c = Case((1,) * 70, tuple(range(0, 140, 2)), 2, 3, 64, seed=5)
    q = c.queries()
    out, lse = c.check(q)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    assert c.dec.kv_attend_rows(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out2, lse=lse2) == B.KV_OK
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "fp4"])
def test_pages_that_are_not_there(kv):
    c = Case((9, 40, 3), (300, 200, 64), 2, 2, 64, types=("bf16", kv), seed=7)
    t = c.table.clone()
    t[0, 3], t[0, 7:12], t[1, 0], t[2, :] = -1, c.n_blocks, -2 ** 31, 2 ** 31 - 1
    out, lse = c.check(table=t)
    assert (out[-3:] == 0).all() and torch.isinf(lse[-3:]).all()
    c.check(table=t, causal=False)


def test_lengths_out_of_range():
    c = Case((5, 5, 40, 4), (100, 64, 70, 32), 1, 2, 64, max_blocks=4, seed=9)
    c.check(lens=torch.tensor([100, -5, 80, 2 ** 31 - 1], dtype=torch.int32))
    c.check(lens=torch.tensor([-2 ** 31, 64, 3, 70], dtype=torch.int32))
    c.check(lens=torch.tensor([2 ** 31 - 1, 64, 3, 70], dtype=torch.int32), causal=False)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp4"), ("fp16", "fp8")], ids="-".join)
def test_what_nobody_sees_makes_no_difference(bad, types):
    """Rows of pages behind the requests' ends, and pages of nobody."""
    c = Case((4, 33, 70), (5, 200, 70), 2, 2, 128, types=types, seed=11)
    seen = torch.zeros((c.n_blocks, c.p), dtype=torch.bool)
    for s, n in enumerate(c.lens.tolist()):
        for t in range(n):
            seen[int(c.table[s, t // c.p]), t % c.p] = True
    q = c.queries()
    want = c.check(q)
    for which in (0, 1):
        c.plane(which)[~seen.cuda()] = bad if types[1] == types[0] else 255 if types[1] == "fp4" else 127
    got = c.check(q)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("x", ["bf16", "fp16"])
def test_odd_values_of_later_tokens(bad, dim, x):
    """Infinities and NaN in keys and values that only some rows of a tile see."""
    c = Case((70, 3), (150, 40), 2, 2, dim, types=(x, x), seed=12)
    q = c.queries()
    for which, t in ((1, 100), (1, 149), (0, 120), (1, 130)):
        c.plane(which)[int(c.table[0, t // c.p]), t % c.p, 1, 3:5] = bad
    out, _ = c.check(q, lse=False)
    assert torch.isfinite(out[:20]).all()


def test_rows_that_see_nothing_behind_odd_values():
    """What one call notes of infinities is nothing to the next one's tiles without a token."""
    c = Case((300, 40), (300, 40), 4, 2, 64, seed=22)
    q = c.queries()
    c.plane(1)[:] = float("inf")
    for _ in range(3):
        out, _ = c.check(q, lse=False)
        assert torch.isinf(out).all()
        none, lse = c.check(q, lens=torch.tensor([0, 0], dtype=torch.int32))
        assert (none == 0).all() and torch.isinf(lse).all()


@pytest.mark.parametrize("x", ["bf16", "fp16"])
def test_the_mean_of_the_largest_values_is_no_infinity(x):
    c = Case((3, 130), (400, 130), 1, 2, 64, types=(x, x), seed=13)
    most = torch.finfo(c.x).max
    c.plane(1)[:] = most
    out, _ = c.check()
    assert (out == most).all()


@pytest.mark.parametrize("scale", [0.0, -0.3, 5.0, 1e-30])
def test_scales(scale):
    Case((20, 70), (300, 100), 1, 3, 64, seed=14).check(scale=scale)


def test_large_scores():
    c = Case((20, 70), (300, 100), 2, 3, 128, seed=15, spread=8.0)
    c.check(c.queries(8.0))


def test_strides_and_orders():
    c = Case((5, 60), (90, 60), 2, 2, 64, seed=16, behind=3)
    q = c.queries()
    want, want_lse = c.check(q)
    r, h, d = q.shape
    wide = torch.zeros((r, 3 * h, d + 8), dtype=c.x, device="cuda")
    wide[:, h:2 * h, :d] = q.cuda()
    table = torch.full((len(c.lens), c.max_blocks + 3), 99, dtype=torch.int32, device="cuda")
    table[:, :c.max_blocks] = c.table.cuda()
    by_head = torch.zeros((h, r, d), dtype=c.x, device="cuda")
    assert c.dec.kv_attend_rows(c.layer, wide[:, h:2 * h, :d], table[:, :c.max_blocks], c.lens.cuda(), by_head.transpose(0, 1),
                                starts=c.starts.cuda()) == B.KV_OK
    assert torch.equal(by_head.transpose(0, 1)[:-3], want[:-3])
    in_place = q.cuda()
    assert c.dec.kv_attend_rows(c.layer, in_place, c.table.cuda(), c.lens.cuda(), in_place, starts=c.starts.cuda()) == B.KV_OK
    assert torch.equal(in_place[:-3], want[:-3])


def test_same_bits_and_other_streams():
    c = Case((16, 3), (5000, 700), 1, 4, 64, seed=17)
    q = c.queries()
    want, lse = c.check(q)
    qd, td, ld, sd = q.cuda(), c.table.cuda(), c.lens.cuda(), c.starts.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side.cuda_stream):
        for _ in range(3):
            out, l2 = torch.empty_like(want), torch.empty_like(lse)
            side.wait_stream(torch.cuda.current_stream())
            assert c.dec.kv_attend_rows(c.layer, qd, td, ld, out, starts=sd, lse=l2, stream=stream) == B.KV_OK
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(l2, lse)


def test_recorded_and_replayed_as_requests_grow():
    """Tables, lengths and rows are read when the kernels run."""
    c = Case((10, 40, 6), (200, 90, 300), 2, 2, 64, seed=18)
    q = c.queries()
    qd, td = q.cuda(), c.table.cuda()
    lens, starts = c.lens.cuda(), c.starts.cuda()
    out, lse = torch.zeros(q.shape, dtype=c.x, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    assert c.dec.kv_attend_rows(c.layer, qd, td, lens, out, starts=starts, lse=lse) == B.KV_OK
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert c.dec.kv_attend_rows(c.layer, qd, td, lens, out, starts=starts, lse=lse) == B.KV_OK
    for new, now in (((10, 40, 6), (200, 90, 300)), ((1, 50, 5), (150, 60, 3)), ((0, 0, 56), (10, 0, 299)), ((20, 20, 16), (190, 88, 250))):
        ls, st = torch.tensor(now, dtype=torch.int32), torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
        lens.copy_(ls)
        starts.copy_(st)
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        ref = R.rows(q, c.values(0), c.values(1), c.table, ls, st, 1 / math.sqrt(c.dim), True, c.n_blocks)
        c.compare(out, lse, ref)


def test_one_decoder_for_many_sizes():
    """Splits of one call leave nothing for the next."""
    c = Case((3, 2, 250), (9000, 40, 250), 1, 4, 64, seed=19)
    q = c.queries()
    for starts, lens in (((0, 3, 5, 255), (9000, 40, 250)), ((0, 1, 2, 3), (8000, 3, 100)), ((0, 3, 5, 255), (9000, 40, 250))):
        c.check(q, starts=torch.tensor(starts, dtype=torch.int32), lens=torch.tensor(lens, dtype=torch.int32))


def test_one_row_is_kv_attend():
    c = Case((1,) * 9, (1, 5, 64, 100, 333, 0, 17, 1000, 4096), 2, 4, 128, seed=20)
    q = c.queries()
    out, lse = c.check(q)
    a, l2 = torch.empty_like(out), torch.empty_like(lse)
    assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), a, lse=l2) == B.KV_OK
    ref = R.rows(q, c.values(0), c.values(1), c.table, c.lens, c.starts, 1 / math.sqrt(c.dim), True, c.n_blocks)
    c.compare(a, l2, ref)


def test_refusals():
    c = Case((3, 4), (20, 30), 2, 2, 64, seed=21)
    q, out = c.queries().cuda(), torch.empty((7, 4, 64), dtype=c.x, device="cuda")
    td, ld, sd = c.table.cuda(), c.lens.cuda(), c.starts.cuda()
    call = lambda *a, **k: c.dec.kv_attend_rows(c.layer, *a, **k)  # noqa: E731
    assert call(q, td, ld, out, starts=sd) == B.KV_OK
    for bad in ((q.float(), td, ld, out), (q[:6], td, ld, out), (q, td[:1], ld, out), (q, td, ld.long(), out), (q, td, ld, out[:, :3]),
                (q.cpu(), td, ld, out), (q, td, ld, None), (None, td, ld, out), (q, td, ld, out.transpose(1, 2))):
        assert call(*bad, starts=sd) == B.KV_EINVAL
    assert call(q, td, ld, out, starts=sd[:2]) == B.KV_EINVAL
    assert call(q, td, ld, out, starts=sd.long()) == B.KV_EINVAL
    assert call(q, td, ld, out) == B.KV_EINVAL                              # seven rows of two requests
    assert call(q, td, ld, out, starts=sd, lse=torch.empty((7, 3), device="cuda")) == B.KV_EINVAL
    assert call(q, td, ld, out, starts=sd, scale=float("nan")) == B.KV_EINVAL
    assert call(q.requires_grad_(), td, ld, out, starts=sd) == B.KV_EINVAL
    with torch.no_grad():
        assert call(q, td, ld, out, starts=sd) == B.KV_OK
    many = torch.empty((8, 4, 64), dtype=c.x, device="cuda")
    assert call(many, td, ld, torch.empty_like(many), starts=sd) == B.KV_E2BIG
    none = D.Decoder(c.cfg, c.cache.data_ptr(), 4, max_seqs=2, max_blocks=c.max_blocks)
    assert none.kv_attend_rows(c.layer, q.detach(), td, ld, out, starts=sd) == B.KV_E2BIG
    v = out._version
    assert call(q.detach(), td, ld, out, starts=sd) == B.KV_OK and out._version == v + 1
