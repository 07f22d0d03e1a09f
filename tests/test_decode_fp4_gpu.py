"""The cache in 4 bits, and heads that are normed on their way into it, against plain 64-bit arithmetic."""
import math

import numpy as np
import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import decode_reference as A
from tests import rows_reference as R
from tests.test_rows_gpu import KIND, X, Case

pytestmark = pytest.mark.gpu

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


# ---- attention of one token over 4 bits -----------------------------------------------------------

def attend(c, q, table=None, lens=None, mass=True):
    table, lens = c.table if table is None else table, c.lens if lens is None else lens
    ref = A.attend(q.double(), c.values(0), c.values(1), table, lens, 1 / math.sqrt(c.dim), c.n_blocks)
    dec = D.Decoder(c.cfg, c.cache.data_ptr(), c.heads * c.group, max_seqs=len(lens), max_blocks=c.max_blocks, x_type=KIND[c.types[0]],
                    kv_type=KIND[c.types[1]])
    n = len(lens)
    out = torch.full(q.shape, float("nan"), dtype=c.x, device="cuda")
    lse = torch.full((n, q.shape[1]), float("nan"), device="cuda")
    before = torch.rand((n, c.max_blocks), generator=c.g).cuda()
    m_out = torch.full_like(before, float("nan")) if mass else None
    assert dec.kv_attend(c.layer, q.cuda(), table.cuda(), lens.cuda(), out, lse=lse, mass=before if mass else None, mass_out=m_out) == B.KV_OK
    torch.cuda.synchronize()
    bound, lse_bound, mass_bound = A.attend_bounds(ref, lens, c.dim, c.x)
    off = (out.cpu().double() - ref["out"]).abs()
    assert (off <= bound).all(), f"out off by {(off / bound).max():.2f} of the bound"
    got, empty = lse.cpu().double(), torch.isinf(ref["lse"])
    assert torch.equal(torch.isinf(got) & (got < 0), empty)
    assert (torch.where(empty, 0.0, (got - ref["lse"]).abs()) <= lse_bound).all()
    if mass:
        off = (m_out.cpu().double() - before.cpu().double() - ref["mass"]).abs()
        assert (off <= mass_bound + 2.0 ** -24 * (before.cpu().double() + ref["mass"])).all()
    return out, lse


def one_token(lens, heads, group, dim, p=16, x="bf16", **kw):
    c = Case((1,) * len(lens), lens, heads, group, dim, p, types=(x, "fp4"), **kw)
    return c, c.queries()


@pytest.mark.parametrize("x", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,group,dim", [(2, 2, 64), (8, 4, 128), (1, 8, 128), (3, 3, 96), (4, 1, 256), (1, 40, 64), (2, 5, 192), (2, 3, 32),
                                             (3, 2, 160), (5, 7, 224), (2, 16, 128), (9, 2, 32)])
def test_heads_and_dimensions(x, heads, group, dim):
    c, q = one_token((1, 33, 100, 0, 64, 17, 130), heads, group, dim, x=x, seed=dim)
    attend(c, q)


@pytest.mark.parametrize("p", [1, 3, 5, 8, 16, 20, 32, 48])
@pytest.mark.parametrize("block_first", [False, True])
def test_block_sizes_and_layouts(p, block_first):
    c, q = one_token((1, 2, 31, 32, 33, 200, 0, 95, 64), 1, 4, 64, p, block_first=block_first, layers=3, layer=2, seed=p)
    attend(c, q)


@pytest.mark.parametrize("n", [1, 15, 31, 32, 33, 65, 257, 1000, 4097, 20011])
@pytest.mark.parametrize("heads,dim", [(1, 128), (8, 64)])
def test_lengths(n, heads, dim):
    c, q = one_token((n,), heads, 4, dim, seed=n)
    attend(c, q)


def test_many_requests():
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 700, 150).tolist()
    c, q = one_token(lens, 2, 4, 128, seed=31)
    attend(c, q)


def test_pages_that_are_not_there():
    c, q = one_token((300, 200, 64), 2, 2, 128, seed=7)
    t = c.table.clone()
    t[0, 3], t[0, 7:12], t[1, 0], t[2, :] = -1, c.n_blocks, -2 ** 31, 2 ** 31 - 1
    out, _ = attend(c, q, table=t)
    assert (out[2] == 0).all()


def test_rows_behind_the_ends_may_hold_anything():
    c, q = one_token((5, 200, 70), 2, 2, 128, seed=11)
    want, _ = attend(c, q)
    seen = torch.zeros((c.n_blocks, c.p), dtype=torch.bool)
    for s, n in enumerate(c.lens.tolist()):
        for t in range(n):
            seen[int(c.table[s, t // c.p]), t % c.p] = True
    for which in (0, 1):
        c.plane(which)[~seen.cuda()] = 255
    assert torch.equal(attend(c, q)[0], want)


@pytest.mark.parametrize("call", ["one", "rows"])
def test_every_number_and_power(call):
    """With one token that is attended to the output is its value: all numbers times all powers that bf16 holds, and NaN."""
    heads, dim = 2, 128
    c, q = one_token((1,) * 128, heads, 1, dim, seed=1)
    rng = np.random.default_rng(1)
    n = heads * dim // 2
    for s in range(128):
        row = torch.from_numpy(rng.integers(0, 256, heads * dim // 32 * 17).astype(np.uint8))
        row[n:] = torch.tensor([(2 * s + j % 2) if 2 * s + j % 2 < 253 else 255 for j in range(n // 16)], dtype=torch.uint8)
        c.plane(1).view(c.n_blocks, c.p, -1)[int(c.table[s, 0]), 0] = row.cuda()
    want = c.values(1)[c.table[:, 0].long(), 0]                               # [request, head, dim]
    out = torch.empty((128, heads, dim), dtype=c.x, device="cuda")
    if call == "one":
        assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out) == B.KV_OK
    else:
        assert c.dec.kv_attend_rows(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out) == B.KV_OK
    got = out.cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    # the weight is one; results below bf16's normal range may be lost
    there = ~want.isnan() & (want.abs() >= 2.0 ** -100)
    assert there.any() and (got[there] - want[there]).abs().le(2.0 ** -8 * want[there].abs()).all()


# ---- new tokens: norms, rotation, 4 bits ----------------------------------------------------------

class Put:
    def __init__(self, new=(3, 1), past=(10, 0), heads=2, group=2, dim=64, p=16, x="bf16", kv="bf16", layers=2, layer=1, block_first=False,
                 rot=None, interleaved=False, axes=1, behind=0, seed=0, norms=(True, True), eps=1e-6, q=True, much=1.0, k_scale=1.0):
        self.g = torch.Generator().manual_seed(seed)
        self.heads, self.dim, self.kv, self.layer, self.block_first, self.eps = heads, dim, kv, layer, block_first, eps
        self.x, self.rot, self.interleaved, self.axes, self.scale = X[x], dim if rot is None else rot, interleaved, axes, k_scale
        q_heads = heads * group
        lens = [a + b for a, b in zip(new, past)]
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
        self.n, n_rows = int(self.starts[-1]), int(self.starts[-1]) + behind
        held = [-(-n // p) for n in lens]
        self.n_blocks, self.p = sum(held) + 3, p
        order = iter(np.random.default_rng(seed).permutation(self.n_blocks).tolist())
        self.table = torch.full((len(lens), max(max(held), 1)), -1, dtype=torch.int32)
        for s, h in enumerate(held):
            for j in range(h):
                self.table[s, j] = next(order)
        head = D.fp4_head_bytes(dim) if kv == "fp4" else dim
        shape = W.KVShape(layers, heads, head, p, self.n_blocks, 1, 1 if kv in ("fp8", "fp4") else 2)
        dims = (self.n_blocks, layers, 2, p, heads, head) if block_first else (layers, 2, self.n_blocks, p, heads, head)
        self.before = (torch.randint(0, 255, dims, generator=self.g).to(torch.uint8) if kv in ("fp8", "fp4")
                       else torch.randn(dims, generator=self.g).to(self.x))
        self.cache = self.before.cuda()
        rand = lambda h: (torch.randn((n_rows, h, dim), generator=self.g) * much).to(self.x)  # noqa: E731
        self.q, self.k, self.v = rand(q_heads) if q else None, rand(heads), rand(heads)
        self.weights = [torch.rand(dim, generator=self.g) + 0.5 if on else None for on in norms]
        pairs = self.rot // 2
        self.sections = (pairs,) if axes == 1 else (pairs // 4, (pairs - pairs // 4) // 2, pairs - pairs // 4 - (pairs - pairs // 4) // 2)
        self.inv_freq = 10000.0 ** -(torch.arange(pairs).float() / max(pairs, 1))
        self.positions = torch.randint(0, 5000, (axes, n_rows), generator=self.g, dtype=torch.int32)
        self.cfg = B.make_config(shape, hbm_layout=1 if block_first else 0)
        self.dec = D.Decoder(self.cfg, self.cache.data_ptr(), q_heads, max_seqs=len(lens), max_blocks=self.table.shape[1], x_type=KIND[x],
                             kv_type=KIND[kv], k_scale=k_scale, v_scale=k_scale, weigh=False)

    def norm(self):
        w = [None if w is None else w.cuda() for w in self.weights]
        return D.HeadNorm(w[0], w[1], self.eps) if any(x is not None for x in w) else None

    def run(self, **kw):
        q = None if self.q is None else self.q.cuda()
        self.q_out = None if q is None else torch.full_like(q, 9.0)
        rope = D.Rope(self.inv_freq.cuda(), self.sections, self.interleaved) if self.rot else None
        rc = self.dec.kv_put(self.layer, self.k.cuda(), self.v.cuda(), self.table.cuda(), self.lens.cuda(), q=q, q_out=self.q_out,
                             starts=self.starts.cuda(), rope=rope, positions=self.positions.cuda() if self.rot else None, norm=self.norm(), **kw)
        assert rc == B.KV_OK, B.kv_strerror(rc)
        torch.cuda.synchronize()

    def want(self, x, weight):
        x = x.double()
        if weight is not None:
            x = R.normed(x, weight, self.eps)
        return A.turned(x, self.positions, self.inv_freq, self.sections, self.rot, self.interleaved) if self.rot else x

    def off(self, x, weight):
        """What 32 bits leave: the mean of squares (dim products and additions), a root, a quotient and two products; angles within
        2^-22, a product each and a sum: of a pair together."""
        size = self.want(x, weight).abs()
        r = self.rot
        both = size.clone()
        i, j = (slice(0, r, 2), slice(1, r, 2)) if self.interleaved else (slice(0, r // 2), slice(r // 2, r))
        both[..., i] = both[..., j] = torch.maximum(size[..., i], size[..., j]) * 1.5
        return ((self.dim / 2 + 8) * 2.0 ** -24 * (weight is not None) + 2.0 ** -21) * both + 1e-38

    def check(self):
        self.run()
        n, u = self.n, HALF_STEP[self.x]
        if self.q is not None:
            got, want = self.q_out.cpu().double(), self.want(self.q, self.weights[0])
            off = self.off(self.q, self.weights[0])
            # (2^-25: half of fp16's smallest number)
            assert ((got - want).abs()[:n] <= (off + u * (want.abs() + off) + 2.0 ** -25)[:n]).all()
            assert (got[n:] == 9.0).all(), "padding was written"
        after = self.cache.cpu()
        touched = torch.zeros((self.n_blocks, self.p), dtype=torch.bool)
        for which, x, weight in ((0, self.k, self.weights[1]), (1, self.v, None)):
            want = self.want(x, weight) if which == 0 else x.double()
            off = self.off(x, weight) if which == 0 else 0 * want
            plane, old = (c[:, self.layer, which] if self.block_first else c[self.layer, which] for c in (after, self.before))
            row = 0
            for s in range(len(self.lens)):
                m = int(self.starts[s + 1] - self.starts[s])
                for i in range(m):
                    t = int(self.lens[s]) - m + i
                    cell = (int(self.table[s, t // self.p]), t % self.p)
                    if 0 <= cell[0] < self.n_blocks:
                        touched[cell] = True
                        self.compare_row(plane[cell], want[row], off[row], f"plane {which} request {s} token {t}")
                    row += 1
            assert torch.equal(plane[~touched], old[~touched]), "rows of other tokens were written"
        other = after.clone()
        if self.block_first:
            other[:, self.layer] = self.before[:, self.layer]
        else:
            other[self.layer] = self.before[self.layer]
        assert torch.equal(other.view(torch.uint8), self.before.view(torch.uint8)), "another layer was written"

    def compare_row(self, got, want, off, what):
        u = HALF_STEP[self.x]
        if self.kv in ("bf16", "fp16"):
            assert ((got.double() - want).abs() <= off + u * (want.abs() + off) + 2.0 ** -25).all(), what
            return
        if self.kv == "fp8":
            g, w = got.view(torch.float8_e4m3fn).double() * self.scale, want.clamp(-448 * self.scale, 448 * self.scale)
            assert ((g - w).abs() <= off + 2.0 ** -4 * (w.abs() + off) + 2.0 ** -10 * self.scale).all(), what
            return
        # 4 bits: the bytes are those of some number within `off`
        g = got.flatten()
        lo, hi = (R.fp4_rows(want.sign() * (want.abs() + d * off).clamp(min=0), self.x) for d in (-1, 1))
        n = self.heads * self.dim // 2
        assert ((g[n:] == lo[n:]) | (g[n:] == hi[n:])).all(), what
        exact = R.fp4_rows(want, self.x)
        same_power = (g[n:] == exact[n:]).repeat_interleave(16)
        v, e, a, b = (R.fp4_values(y, self.heads, self.dim).flatten() for y in (g, exact, lo, hi))
        power = torch.exp2(g[n:].double() - 127).repeat_interleave(32)
        # off by no more than half a step and the bound wherever the power is the exact one's (6 stands for what is above, too)
        w, o = want.flatten(), off.flatten()
        step = torch.where(v.abs() >= 4 * power, 2.0, torch.where(v.abs() >= 2 * power, 1.0, 0.5)) * power
        ok = ((v - w).abs() <= step / 2 + o) | ((v.abs() == 6 * power) & (w.abs() >= 5 * power - o))
        assert ok.all(), what
        if not off.any():
            assert torch.equal(g, exact), what
        assert ((v == e) | ~same_power.repeat_interleave(2) | (v == a) | (v == b)).all(), what


@pytest.mark.parametrize("x,kv", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp8"), ("fp16", "fp8"), ("bf16", "fp4"), ("fp16", "fp4")])
@pytest.mark.parametrize("heads,group,dim,rot,interleaved", [(2, 2, 64, 64, False), (8, 4, 128, 128, False), (1, 8, 128, 64, False),
                                                             (3, 3, 96, 96, True), (4, 1, 256, 256, False), (2, 5, 192, 96, True),
                                                             (2, 3, 32, 16, False), (3, 2, 160, 40, False), (1, 1, 32, 8, False),
                                                             (5, 7, 224, 200, False), (2, 2, 96, 24, True), (2, 2, 64, 0, False)])
def test_put_heads_and_rotations(x, kv, heads, group, dim, rot, interleaved):
    Put((3, 1, 0, 20), (10, 0, 7, 90), heads, group, dim, x=x, kv=kv, rot=rot, interleaved=interleaved, behind=2, seed=dim + rot,
        k_scale=0.02 if kv == "fp8" else 1.0).check()


@pytest.mark.parametrize("x,kv", [("bf16", "bf16"), ("fp16", "fp8")])
@pytest.mark.parametrize("dim,rot", [(40, 40), (80, 40), (8, 8), (104, 72), (72, 56), (200, 8)])
def test_put_norms_of_other_dimensions(x, kv, dim, rot):
    for interleaved in (False, True):
        Put((2, 5), (30, 0), 3, 2, dim, p=5, x=x, kv=kv, rot=rot, interleaved=interleaved, seed=dim).check()


@pytest.mark.parametrize("norms", [(True, False), (False, True), (False, False)])
def test_put_some_norms(norms):
    Put((4, 9), (0, 50), 2, 4, 128, kv="fp4", norms=norms, seed=1).check()
    if any(norms):
        Put((4, 9), (0, 50), 2, 4, 128, norms=norms, seed=1).check()


@pytest.mark.parametrize("kv", ["bf16", "fp4"])
def test_put_without_q_over_axes_and_blocks_first(kv):
    Put((4, 9), (3, 50), 2, 4, 128, kv=kv, norms=(False, True), q=False, axes=3, block_first=True, p=5, layers=3, seed=2).check()


@pytest.mark.parametrize("rows", [1, 63, 1025])
def test_put_many_rows(rows):
    Put((rows,), (17,), 2, 2, 32, kv="fp4", seed=rows).check()
    Put((rows,), (17,), 2, 2, 32, seed=rows).check()


@pytest.mark.parametrize("much", [1e-30, 1e-5, 300.0, 1e18])
def test_put_small_and_large_values(much):
    Put((5,), (3,), 2, 2, 64, kv="fp4", norms=(False, False), much=much, seed=5).check()
    Put((5,), (3,), 2, 2, 64, kv="fp4", much=much, seed=5).check()


def test_put_values_of_4_bits_exactly():
    """Middles between numbers, zeros, the largest, and groups with infinities or NaN."""
    c = Put((8,), (3,), 2, 1, 64, kv="fp4", norms=(False, False), rot=0, seed=6)
    grid = torch.tensor([0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.5, 6.0, 6.5, 7.0, 7.5, 7.96875, 4.0])
    for x in (c.k, c.v):
        for r in range(8):
            x[r] = (grid.repeat(4) * 2.0 ** (r * 30 - 110)).to(c.x) * (-1) ** r
        x[6, 1, 40], x[7, 0, 0], x[5, 0, 33:35] = float("nan"), float("inf"), -float("inf")
        x[4, 1], x[3, 0, :32] = 0.0, torch.finfo(c.x).max
    c.run()
    at = c.cache.cpu()[c.layer]
    for which, x in ((0, c.k), (1, c.v)):
        for r in range(8):
            t = 3 + r
            got = at[which][int(c.table[0, t // c.p]), t % c.p].flatten()
            assert torch.equal(got, R.fp4_rows(x[r].double(), c.x)), (which, r)


def test_put_fp16_powers_stay_where_fp16_holds_the_numbers():
    c = Put((3,), (0,), 1, 1, 32, x="fp16", kv="fp4", norms=(False, False), rot=0, seed=7)
    c.k[0], c.k[1], c.k[2] = 65504.0, 2.0 ** -24, 0.0
    c.run()
    at = c.cache.cpu()[c.layer][0]
    for r in range(3):
        assert torch.equal(at[int(c.table[0, 0]), r].flatten(), R.fp4_rows(c.k[r].double(), c.x))


def test_put_bad_pages_and_tokens():
    for kv in ("bf16", "fp4"):
        c = Put((4, 20, 5), (20, 10, 0), 2, 2, 64, kv=kv, seed=8)
        c.table[0, 1], c.table[1, 0] = c.n_blocks, -7
        c.check()
        c.lens[2] = 3                    # five rows of a request of three tokens: the first two have no place
        c.cache.copy_(c.before)
        c.run()
        want = c.want(c.q, c.weights[0])
        assert ((c.q_out.cpu().double() - want).abs() <= c.off(c.q, c.weights[0]) + 2.0 ** -8 * want.abs() * 1.01).all()


def test_norms_leave_the_other_path_as_it_is():
    """Weights of one and heads whose mean square is one: the norm changes nothing beyond its roundings."""
    c = Put((4, 9), (0, 50), 2, 4, 128, seed=9, eps=0.0)
    c.weights = [torch.ones(128)] * 2
    c.q, c.k = (x.sign().to(c.x) for x in (c.q, c.k))
    c.run()
    q, cache = c.q_out.clone(), c.cache.clone()
    c.weights = [None, None]
    c.cache.copy_(c.before)
    c.run()
    assert (q.double() - c.q_out.double()).abs().max() <= 2.0 ** -7 and (cache.double() - c.cache.double()).abs().max() <= 2.0 ** -7


def test_put_replayed():
    c = Put((5, 3), (10, 0), 2, 2, 64, kv="fp4", seed=10)
    c.run()
    want, want_q = c.cache.clone(), c.q_out.clone()
    norm, rope = c.norm(), D.Rope(c.inv_freq.cuda(), c.sections)
    q, k, v, table, lens, starts, pos = (x.cuda() for x in (c.q, c.k, c.v, c.table, c.lens, c.starts, c.positions))
    out = torch.full_like(q, 9.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert c.dec.kv_put(c.layer, k, v, table, lens, q=q, q_out=out, starts=starts, rope=rope, positions=pos, norm=norm) == B.KV_OK
    for _ in range(3):
        c.cache.copy_(c.before)
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.cache, want) and torch.equal(out, want_q)


def test_refusals():
    c = Put((4, 9), (0, 50), 2, 4, 64, seed=11)
    w = torch.ones(64, device="cuda")
    args = (c.layer, c.k.cuda(), c.v.cuda(), c.table.cuda(), c.lens.cuda())
    kw = dict(q=c.q.cuda(), q_out=c.q.cuda(), starts=c.starts.cuda())
    assert c.dec.kv_put(*args, norm=D.HeadNorm(w, w), **kw) == B.KV_OK
    assert c.dec.kv_put(*args, norm=D.HeadNorm(w[:32].clone(), w), **kw) == B.KV_EINVAL
    assert c.dec.kv_put(*args, norm=D.HeadNorm(w, w), starts=kw["starts"]) == B.KV_EINVAL       # a weight for q, and no q
    wide = torch.ones(68, device="cuda")
    assert c.dec.kv_put(*args, norm=D.HeadNorm(None, wide[1:65]), **kw) == B.KV_EUNSUP
    assert c.dec.kv_put(*args, norm=D.HeadNorm(w.clone().requires_grad_(), w), **kw) == B.KV_EINVAL
    for bad in (dict(q_weight=w.half(), k_weight=None), dict(q_weight=None, k_weight=w.cpu()), dict(q_weight=w, k_weight=w, eps=-1.0),
                dict(q_weight=w, k_weight=w, eps=float("nan"))):
        with pytest.raises(ValueError):
            D.HeadNorm(**bad)
    for dim in (0, 16, 40, -32):
        with pytest.raises(ValueError):
            D.fp4_head_bytes(dim)
    shape = W.KVShape(1, 2, 64, 16, 4, 1, 1)       # 64 bytes of a head are no 17ths
    cache = torch.zeros(shape.cache_dims(), dtype=torch.uint8, device="cuda")
    with pytest.raises(B.KVError):
        D.Decoder(B.make_config(shape), cache.data_ptr(), 2, 1, 1, kv_type=B.KV_FP4)


def test_a_run_of_them(seed=12):
    """A prompt, its attention, decode steps, all over one cache in 4 bits with normed heads: put, rows, put, one token."""
    heads, group, dim, p, n = 2, 4, 128, 16, 3
    new = (37, 5, 130)
    c = Put(new, (0, 0, 0), heads, group, dim, p, kv="fp4", seed=seed)
    c.table = torch.full((n, 12), -1, dtype=torch.int32)
    blocks = iter(range(c.n_blocks))
    for s in range(n):
        for j in range(-(-new[s] // p)):
            c.table[s, j] = next(blocks)
    dec = D.Decoder(c.cfg, c.cache.data_ptr(), heads * group, max_seqs=n, max_blocks=12, kv_type=B.KV_FP4, max_rows=sum(new))
    norm, rope = c.norm(), D.Rope(c.inv_freq.cuda(), c.sections)
    table, lens, starts = c.table.cuda(), c.lens.cuda(), c.starts.cuda()
    q = c.q.cuda()
    out = torch.empty_like(q)
    assert dec.kv_put(c.layer, c.k.cuda(), c.v.cuda(), table, lens, q=q, q_out=q, starts=starts, rope=rope, norm=norm) == B.KV_OK
    assert dec.kv_attend_rows(c.layer, q, table, lens, out, starts=starts) == B.KV_OK
    torch.cuda.synchronize()
    plane = lambda i: R.fp4_values(c.cache[c.layer, i].cpu().flatten(-2), heads, dim)  # noqa: E731
    ref = R.rows(q.cpu(), plane(0), plane(1), c.table, c.lens, c.starts, 1 / math.sqrt(dim), True, c.n_blocks)
    bound, _ = R.rows_bounds(ref, dim, c.x)
    assert ((out.cpu().double() - ref["out"]).abs() <= bound).all()
    for step in range(3):
        lens += 1
        room = c.lens + step + 1
        assert all(int(c.table[s, (int(room[s]) - 1) // p]) >= 0 for s in range(n))
        g = torch.Generator().manual_seed(step)
        q1, k1, v1 = (torch.randn((n, h, dim), generator=g).to(c.x).cuda() for h in (heads * group, heads, heads))
        o1 = torch.empty_like(q1)
        assert dec.kv_put(c.layer, k1, v1, table, lens, q=q1, q_out=q1, rope=rope, norm=norm) == B.KV_OK
        assert dec.kv_attend(c.layer, q1, table, lens, o1) == B.KV_OK
        torch.cuda.synchronize()
        ref = A.attend(q1.cpu().double(), plane(0), plane(1), c.table, room, 1 / math.sqrt(dim), c.n_blocks)
        assert ((o1.cpu().double() - ref["out"]).abs() <= A.attend_bounds(ref, room, dim, c.x)[0]).all()
