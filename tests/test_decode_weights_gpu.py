"""What attention's weights are when they meet the values: enough digits that a result is off by its own rounding
and little else, and no weight of 0 beside a value of infinity."""
import math

import pytest
import torch

from tests import decode_reference as R
from tests.test_decode_gpu import ALL_TYPES, Case

pytestmark = pytest.mark.gpu


def bound(ref, lens, dim, types, x):
    """A score is off by e = (dim + 4) 2^-24 size and twice 2^-24 of what it is compared with; a weight by twice that,
    by eight steps of exp2 and log2 of 2^-22, and by a rounding of the sums per 32 tokens and 64 in the joins; as it meets
    V by 2^-15, 2^-21, or twice 2^-11 (8-bit cache and bf16: numerator and sum) of itself and 2^-35 of the largest; the
    result by half a step."""
    half = R.HALF_STEP[x]
    digits = 2.0 ** -21 if x == torch.float16 else 2.0 ** -10 * (1 + 2.0 ** -10) if types[1] == "fp8" else 2.0 ** -15
    steps = (lens.double() / 32 + 64)[:, None]
    e = (dim + 4) * R.U32 * ref["size"] + 4 * R.U32 * (ref["size"] + 1)
    rel = 2 * (e + 8 * 2.0 ** -22 + steps * R.U32) + digits
    few = (lens.double() * 2.0 ** -35)[:, None] * ref["top"]
    off = (rel * (1 + 2.0 ** -7))[..., None] * ref["spread"] + few[..., None]
    return off + half * (ref["out"].abs() + off) + (2.0 ** -25 if x == torch.float16 else 2.0 ** -133)


@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
@pytest.mark.parametrize("lens,heads,group,dim", [((2, 3, 5, 9, 16, 33), 2, 4, 64), ((40, 7, 100, 20), 2, 3, 40), ((700, 3000, 64), 2, 8, 128),
                                                  ((20, 200), 2, 2, 256), ((5, 90, 31), 1, 24, 96)])
def test_a_result_is_off_by_its_own_rounding(types, lens, heads, group, dim):
    c = Case(heads, group, dim, lens=lens, types=types, seed=dim, k_scale=0.02 if types[1] == "fp8" else 1.0,
             v_scale=0.01 if types[1] == "fp8" else 1.0)
    q = c.queries()
    ref = R.attend(q.double(), c.values(0), c.values(1), c.table, c.lens, 1 / math.sqrt(dim), c.n_blocks)
    out = torch.empty(q.shape, dtype=c.x, device="cuda")
    assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out) == 0
    off, most = (out.cpu().double() - ref["out"]).abs(), bound(ref, c.lens, dim, types, c.x)
    assert (off <= most).all(), f"off by {(off / most).max():.2f} of the bound"


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp16")], ids="-".join)
@pytest.mark.parametrize("n,p", [(20, 16), (300, 5), (9000, 16)])
@pytest.mark.parametrize("below", [0, 28, 60])
def test_a_value_of_infinity_stays_one(types, n, p, below):
    """Under a weight of 2^-40 or 2^-86 of the largest, and under one that a 16-bit number holds exactly; both signs
    together are NaN; other dimensions do not see it."""
    c = Case(1, 2, 64, p, lens=(n,), types=types, seed=n + below)
    k, v = c.plane(0), c.plane(1)
    at = [(int(c.table[0, t // p]), t % p) for t in range(n)]
    k.fill_(0.0)
    for t in range(0, n, 3):
        k[at[t]] = -below / 64              # scores of -below beside scores of 0
    q, table, lens = torch.ones((1, 2, 64), dtype=c.x).cuda(), c.table.cuda(), c.lens.cuda()
    want, got = torch.empty_like(q), torch.empty_like(q)
    assert c.dec.kv_attend(c.layer, q, table, lens, want, scale=1.0) == 0 and torch.isfinite(want).all()
    light, heavy = n // 2 // 3 * 3, 7
    v[at[light]][..., 5] = float("inf")
    v[at[light]][..., 6] = float("-inf")
    v[at[heavy]][..., 9] = float("-inf")
    v[at[light]][..., 11] = float("inf")
    v[at[heavy]][..., 11] = float("-inf")
    assert c.dec.kv_attend(c.layer, q, table, lens, got, scale=1.0) == 0
    assert torch.isposinf(got[..., 5]).all() and torch.isneginf(got[..., 6]).all() and torch.isneginf(got[..., 9]).all()
    assert got[..., 11].isnan().all()
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[[5, 6, 9, 11]] = False
    assert torch.equal(got[..., rest], want[..., rest])


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp16")], ids="-".join)
@pytest.mark.parametrize("n", [40, 9000])
def test_scores_of_minus_infinity_weigh_nothing(types, n):
    """Not even beside the largest values there are, and many of them."""
    c = Case(1, 2, 64, lens=(n,), types=types, seed=n)
    k, v = c.plane(0), c.plane(1)
    q = (c.queries().abs() + 0.25).cuda()
    table, lens = c.table.cuda(), c.lens.cuda()
    some = torch.tensor([t for t in range(n) if t % 3], device="cuda")
    page, row = table[0, some // 16].long(), some % 16
    k[page, row] = 0.0
    k[page, row, :, 0] = float("-inf")
    want, got = torch.empty_like(q), torch.empty_like(q)
    v[page, row] = 0.0
    assert c.dec.kv_attend(c.layer, q, table, lens, want) == 0 and torch.isfinite(want).all()
    v[page, row] = torch.finfo(c.x).max
    assert c.dec.kv_attend(c.layer, q, table, lens, got) == 0
    assert torch.equal(got, want)


@pytest.mark.parametrize("v_scale", [1e-38, 1e-30, 1e35])
@pytest.mark.parametrize("lens", [(9000, 5), (40, 3)])
def test_scales_near_the_ends_of_what_a_float_holds(v_scale, lens):
    """Nothing on the way to a result that bf16 holds is too small or too large for 32 bits."""
    types = ("bf16", "fp8")
    c = Case(1, 2, 64, lens=lens, types=types, seed=51, k_scale=0.02, v_scale=v_scale)
    c.plane(1).copy_(torch.randint(0, 0x7F, c.plane(1).shape, generator=c.g, dtype=torch.uint8))     # none below 0: results are no less
    q = c.queries()
    ref = R.attend(q.double(), c.values(0), c.values(1), c.table, c.lens, 0.125, c.n_blocks)
    out = torch.empty(q.shape, dtype=c.x, device="cuda")
    assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out) == 0
    off, most = (out.cpu().double() - ref["out"]).abs(), bound(ref, c.lens, 64, types, c.x)
    assert (off <= most).all(), f"off by {(off / most).max():.2f} of the bound"


@pytest.mark.parametrize("types", ALL_TYPES, ids="-".join)
@pytest.mark.parametrize("lens", [(2, 40, 1), (5000, 300)])
def test_the_largest_values_have_a_mean(types, lens):
    """Sums over tokens stay within 32 bits where every value is the type's largest, or half of it."""
    c = Case(2, 2, 64, lens=lens, types=types, seed=52)
    top = 448.0 if types[1] == "fp8" else torch.finfo(c.x).max
    for dims, value in ((slice(0, 32), top), (slice(32, 64), -top / 2)):
        to = c.plane(1)[..., dims]
        to.copy_(torch.full(to.shape, value).to(torch.float8_e4m3fn).view(torch.uint8) if types[1] == "fp8" else torch.full(to.shape, value))
    for much in (0.0, 1.0):
        q = c.queries(much).cuda()
        out = torch.empty_like(q)
        assert c.dec.kv_attend(c.layer, q, c.table.cuda(), c.lens.cuda(), out) == 0
        assert (out[..., :32] == top).all() and (out[..., 32:] == -top / 2).all()
