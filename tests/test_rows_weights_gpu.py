"""What the weights of attention of many rows are when they meet the values."""
import math

import pytest
import torch

from paper_2601_20309_amd import binding as B
from tests import rows_reference as R
from tests.test_rows_gpu import Case

pytestmark = pytest.mark.gpu


def bound(ref, dim, x, digits):
    """A score is off by e = (dim + 4) 2^-24 size and twice 2^-24 of what it is compared with; a weight by twice that (numerator and
    sum), by eight steps of exp2 and log2 of 2^-22, and by a rounding of the sums for each token and 64 in the joins; as it meets V by
    `digits` of itself and 2^-36 of the largest; the result by half a step."""
    e = (dim + 4) * R.U32 * ref["size"] + 4 * R.U32 * (ref["size"] + 1)
    rel = 2 * (e + 8 * 2.0 ** -22 + (ref["tokens"][:, None] + 64) * R.U32) + digits
    few = (ref["tokens"][:, None] * 2.0 ** -36) * ref["top"]
    off = (rel * (1 + 2.0 ** -7))[..., None] * ref["spread"] + few[..., None]
    half = R.HALF_STEP[x]
    return off + half * (ref["out"].abs() + off) + (2.0 ** -25 if x == torch.float16 else 2.0 ** -133)


@pytest.mark.parametrize("x", ["bf16", "fp16"])
@pytest.mark.parametrize("new,lens,heads,group,dim", [((2, 9, 5, 16), (2, 9, 5, 33), 2, 4, 64), ((40, 7, 100), (40, 50, 100), 3, 3, 40),
                                                      ((130, 3), (700, 64), 2, 8, 128), ((20, 60), (20, 200), 2, 2, 256),
                                                      ((1200,), (1300,), 32, 1, 64)])
def test_beside_8_bits_a_result_is_off_by_its_own_rounding(x, new, lens, heads, group, dim):
    """Weights are fp16 numbers whatever the outputs' type: values in 8 bits are, too."""
    c = Case(new, lens, heads, group, dim, types=(x, "fp8"), seed=dim, k_scale=0.02, v_scale=0.01)
    q = c.queries()
    ref = R.rows(q, c.values(0), c.values(1), c.table, c.lens, c.starts, 1 / math.sqrt(dim), True, c.n_blocks)
    out = torch.empty(q.shape, dtype=c.x, device="cuda")
    assert c.dec.kv_attend_rows(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out, starts=c.starts.cuda()) == B.KV_OK
    off, most = (out.cpu().double() - ref["out"]).abs(), bound(ref, dim, c.x, 2.0 ** -11)
    assert (off <= most).all(), f"off by {(off / most).max():.2f} of the bound"


@pytest.mark.parametrize("v_scale", [1e-38, 1e-30, 1e35])
@pytest.mark.parametrize("new,lens", [((3, 5), (9000, 5)), ((130,), (2000,))])
def test_scales_near_the_ends_of_what_a_float_holds(v_scale, new, lens):
    """Nothing on the way to a result that bf16 holds is too small or too large for 32 bits."""
    c = Case(new, lens, 1, 2, 64, types=("bf16", "fp8"), seed=51, k_scale=0.02, v_scale=v_scale)
    c.plane(1).copy_(torch.randint(0, 0x7F, c.plane(1).shape, generator=c.g, dtype=torch.uint8))
    q = c.queries()
    ref = R.rows(q, c.values(0), c.values(1), c.table, c.lens, c.starts, 0.125, True, c.n_blocks)
    out = torch.empty(q.shape, dtype=c.x, device="cuda")
    assert c.dec.kv_attend_rows(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out, starts=c.starts.cuda()) == B.KV_OK
    off, most = (out.cpu().double() - ref["out"]).abs(), bound(ref, 64, c.x, 2.0 ** -11)
    assert (off <= most).all(), f"off by {(off / most).max():.2f} of the bound"


@pytest.mark.parametrize("x,below", [("bf16", 0), ("bf16", 28), ("bf16", 60), ("fp16", 0), ("fp16", 12), ("fp16", 24)])
@pytest.mark.parametrize("new,n,heads,group", [(3, 20, 1, 2), (3, 9000, 1, 2), (130, 300, 1, 2), (130, 5000, 1, 2), (1300, 1700, 32, 2)])
def test_a_value_of_infinity_stays_one(x, below, new, n, heads, group):
    """Under weights of 2^-86 (bf16) and 2^-34 (fp16) of the largest, and under one that a 16-bit number holds exactly, in a tile that all rows
    see and in the last one; both signs together are NaN; other dimensions do not see it, and neither do rows before it."""
    c = Case((new,), (n,), heads, group, 64, types=(x, x), seed=n + below)
    k, v = c.plane(0), c.plane(1)
    at = lambda t: (int(c.table[0, t // c.p]), t % c.p)  # noqa: E731
    k.fill_(0.0)
    for t in range(0, n, 3):
        k[at(t)] = -below / 64              # scores of -below beside scores of 0
    q, table, lens, starts = torch.ones((new, heads * group, 64), dtype=c.x).cuda(), c.table.cuda(), c.lens.cuda(), c.starts.cuda()
    want, got = torch.empty_like(q), torch.empty_like(q)
    call = lambda out: c.dec.kv_attend_rows(c.layer, q, table, lens, out, starts=starts, scale=1.0)  # noqa: E731
    assert call(want) == B.KV_OK and torch.isfinite(want).all()
    first, last, heavy = (n - new) // 2 // 3 * 3, (n - 2) // 3 * 3, 7
    v[at(first)][..., 5] = float("inf")
    v[at(first)][..., 6] = float("-inf")
    v[at(heavy)][..., 9] = float("-inf")
    v[at(first)][..., 11] = float("inf")
    v[at(heavy)][..., 11] = float("-inf")
    v[at(last)][..., 13] = float("-inf")
    assert call(got) == B.KV_OK
    assert torch.isposinf(got[..., 5]).all() and torch.isneginf(got[..., 6]).all() and torch.isneginf(got[..., 9]).all()
    assert got[..., 11].isnan().all()
    before = last - (n - new)               # rows that do not see the last one
    assert torch.isneginf(got[before:, :, 13]).all() and torch.equal(got[:before, :, 13], want[:before, :, 13])
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[[5, 6, 9, 11, 13]] = False
    assert torch.equal(got[..., rest], want[..., rest])
