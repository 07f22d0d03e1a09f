"""Means of the largest values there are: no sum on the way to them is beyond 32 bits, however many tokens there are and however their
scores rise."""
import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import rows_reference as R
from tests.test_rows_gpu import Case
from tests.test_rows_weights_gpu import bound

pytestmark = pytest.mark.gpu

KIND = {"bf16": B.KV_BF16, "fp16": B.KV_FP16, "fp4": B.KV_FP4}
X = {"bf16": torch.bfloat16, "fp16": torch.float16}
P = 16


def largest_values(types, heads, dim, scores):
    """A cache of one layer whose tokens give these scores (to base e) to a query of ones, in pages of 16; values are the largest, the second
    half of dimensions half of it below 0.  Returns it, its config, and the two numbers."""
    x, fp4 = X[types[0]], types[1] == "fp4"
    n = -(-len(scores) // P)
    shape = W.KVShape(1, heads, D.fp4_head_bytes(dim) if fp4 else dim, P, n, 1, 1 if fp4 else 2)
    if fp4:
        # a key has one number, 4 or nothing, times a power; of values all are 6 and -3 times the highest power
        top = 6.0 * 2.0 ** (125 if x == torch.bfloat16 else 13)
        cache = torch.zeros((1, 2, n * P, heads * dim // 2 + heads * dim // 32), dtype=torch.uint8)
        bytes_ = heads * dim // 2
        codes = torch.full((heads, dim // 2), 7 | 7 << 4, dtype=torch.uint8)
        codes[:, dim // 4:] = 13 | 13 << 4
        cache[0, 1, :, :bytes_], cache[0, 1, :, bytes_:] = codes.flatten(), 127 + (125 if x == torch.bfloat16 else 13)
        cache[0, 0, :, bytes_:] = 127
        assert set(scores) <= {0.0, 4.0}
        for h in range(heads):
            cache[0, 0, :len(scores), h * dim // 2] = torch.tensor([6 if s else 0 for s in scores], dtype=torch.uint8)
        cache = cache.view(1, 2, n, P, -1)
    else:
        top = float(torch.finfo(x).max)
        cache = torch.zeros((1, 2, n * P, heads, dim), dtype=x)
        cache[0, 0, :len(scores), :, 0] = torch.tensor(scores).to(x)[:, None]
        cache[0, 1, :, :, :dim // 2], cache[0, 1, :, :, dim // 2:] = top, -top / 2
        cache = cache.view(1, 2, n, P, heads, dim)
    return cache.cuda(), B.make_config(shape), top


def decoder(types, cache, cfg, heads, group, **kw):
    return D.Decoder(cfg, cache.data_ptr(), heads * group, x_type=KIND[types[0]], kv_type=KIND[types[1]], weigh=False, **kw)


ALL = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp4"), ("fp16", "fp4")]


def are_means(out, top):
    """Half a step for the weights as they meet the values, and half a step for the result: a step in all, 2^-10 of it more for sums in
    32 bits."""
    want = torch.full((out.shape[-1],), top, dtype=torch.float64, device=out.device)
    want[out.shape[-1] // 2:] = -top / 2
    assert ((out.double() - want).abs() <= torch.finfo(out.dtype).eps * (1 + 2.0 ** -10) * want.abs()).all()


@pytest.mark.parametrize("types", ALL, ids="-".join)
@pytest.mark.parametrize("call", ["one", "rows of 32", "rows of 128", "rows of 256"])
@pytest.mark.parametrize("score", [5.1875, 2.0, 40.0])
def test_scores_rise_behind_the_first_tokens(types, call, score):
    """All requests have the same pages: the first 256 tokens have scores of 0 and the others higher ones (7.5, 2.9 and 58 to base 2).  So many
    requests that a wave has hundreds of tokens of one."""
    heads, dim, n = 8, 64, 4000
    group, new, seqs = {"one": (4, 1, 300), "rows of 32": (4, 2, 64), "rows of 128": (4, 100, 20), "rows of 256": (4, 300, 40)}[call]
    if types[1] == "fp4":
        score = 4.0
    cache, cfg, top = largest_values(types, heads, dim, [0.0 if t < 256 else score for t in range(n)])
    dec = decoder(types, cache, cfg, heads, group, max_seqs=seqs, max_blocks=n // P, max_rows=0 if call == "one" else seqs * new)
    table = torch.arange(n // P, dtype=torch.int32, device="cuda").expand(seqs, -1).contiguous()
    lens = torch.full((seqs,), n, dtype=torch.int32, device="cuda")
    q = torch.ones((seqs * new, heads * group, dim), dtype=X[types[0]], device="cuda")
    out = torch.empty_like(q)
    if call == "one":
        assert dec.kv_attend(0, q, table, lens, out, scale=1.0) == B.KV_OK
    else:
        starts = torch.arange(0, seqs * new + 1, new, dtype=torch.int32, device="cuda")
        assert dec.kv_attend_rows(0, q, table, lens, out, starts=starts, scale=1.0) == B.KV_OK
    are_means(out, top)


@pytest.mark.parametrize("types", ALL, ids="-".join)
@pytest.mark.parametrize("call,new", [("one", 1), ("rows", 1), ("rows", 64), ("rows", 300)])
def test_more_tokens_than_a_small_weight_makes_up_for(types, call, new):
    """300 000 tokens with the same score, of one page that a request has again and again."""
    heads, group, dim, n = 2, 4, 64, 300_000
    cache, cfg, top = largest_values(types, heads, dim, [0.0] * P)
    blocks = n // P
    dec = decoder(types, cache, cfg, heads, group, max_seqs=1, max_blocks=blocks, max_rows=new if call == "rows" else 0)
    table = torch.zeros((1, blocks), dtype=torch.int32, device="cuda")
    lens = torch.full((1,), n, dtype=torch.int32, device="cuda")
    q = torch.ones((new, heads * group, dim), dtype=X[types[0]], device="cuda")
    out = torch.empty_like(q)
    if call == "one":
        assert dec.kv_attend(0, q, table, lens, out, scale=1.0) == B.KV_OK
    else:
        starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        assert dec.kv_attend_rows(0, q, table, lens, out, starts=starts, scale=1.0) == B.KV_OK
    are_means(out, top)


@pytest.mark.parametrize("call", ["one", "rows"])
@pytest.mark.parametrize("n", [40, 100, 5000])
@pytest.mark.parametrize("power", [-60, -100, -110, -115])
def test_small_values_are_not_lost(call, n, power):
    """Room for the largest values is no more than they take: those near the other end of bf16 are as exact as others.  A sum in 32 bits is
    off by 2^-150 for each of its steps of 16 tokens (and 64 in the joins), beside weights that add up to 2^-16 and more, times the share
    that meets the values, 2^-6 in a decoder of 5000 tokens."""
    c = Case((1,), (n,), 2, 4, 64, seed=n)
    c.plane(1).mul_(2.0 ** power)
    q = c.queries()
    ref = R.rows(q, c.values(0), c.values(1), c.table, c.lens, c.starts, 0.125, True, c.n_blocks)
    out = torch.empty(q.shape, dtype=c.x, device="cuda")
    if call == "one":
        assert c.dec.kv_attend(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out, scale=0.125) == B.KV_OK
    else:
        assert c.dec.kv_attend_rows(c.layer, q.cuda(), c.table.cuda(), c.lens.cuda(), out, starts=c.starts.cuda(), scale=0.125) == B.KV_OK
    most = bound(ref, 64, c.x, 2.0 ** -15 if call == "one" else 2.0 ** -8) - 2.0 ** -36 * n * ref["top"][..., None]
    most = most + (n / 16 + 64) * 2.0 ** -150 * 2.0 ** 16 * (2.0 ** 6 if n > 128 else 1.0)
    off = (out.cpu().double() - ref["out"]).abs()
    assert (off <= most).all(), f"off by {(off / most).max():.2f} of the bound"
