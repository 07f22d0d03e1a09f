"""Attention of many rows and the cache in 4 bits at sizes that take other ways: tiles of 256 rows, requests by the thousand, pages
beyond 4 GiB."""
import math

import numpy as np
import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import decode_reference as A
from tests import rows_reference as R
from tests.test_decode_fp4_gpu import Put
from tests.test_rows_gpu import KIND, X, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types,heads,group,dim,causal", [(("bf16", "bf16"), 64, 1, 64, True), (("fp16", "fp16"), 4, 8, 128, True),
                                                          (("bf16", "fp8"), 2, 17, 96, False), (("bf16", "fp4"), 16, 3, 64, True)])
def test_tiles_of_256_rows(types, heads, group, dim, causal):
    """So many rows to each request that 256 go to a workgroup; some pages are not there."""
    new = (66000 // (heads * group) + 1100 // group, 3)
    c = Case(new, (new[0] + 130, 70), heads, group, dim, types=types, seed=heads, behind=2)
    c.table[0, 5] = -1
    c.check(causal=causal)


def test_tiles_of_256_rows_and_odd_values():
    c = Case((1100,), (1300,), 64, 1, 64, seed=77)
    for which, t, bad in ((1, 400, float("nan")), (1, 1200, float("inf")), (0, 800, float("nan")), (1, 1299, -float("inf"))):
        c.plane(which)[int(c.table[0, t // c.p]), t % c.p, 3, 5:9] = bad
    out, _ = c.check(lse=False)
    assert torch.isfinite(out[:199]).all()


def test_thousands_of_requests():
    rng = np.random.default_rng(6)
    n = 4300
    new = (rng.random(n) < 0.4).astype(int)
    lens = rng.integers(0, 12, n)
    lens[4000], new[4000] = 700, 60
    c = Case(new.tolist(), lens.tolist(), 1, 2, 64, p=8, seed=6)
    c.check()
    c.check(causal=False)


def test_put_for_many_requests():
    rng = np.random.default_rng(7)
    new, past = rng.integers(0, 4, 70), rng.integers(0, 30, 70)
    for kv in ("bf16", "fp4"):
        Put(tuple(new), tuple(past), 1, 2, 64, kv=kv, seed=7, behind=3).check()
        Put(tuple(new[:64]), tuple(past[:64]), 1, 2, 64, kv=kv, seed=8, behind=3).check()


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "fp8"), ("fp16", "fp4")], ids="-".join)
def test_pages_beyond_4_gib(types):
    """The same pages, and the last ones of a cache whose planes have 5 GiB each."""
    heads, dim, p, x = 8, 128, 16, X[types[0]]
    c = Case((40, 3, 1), (300, 50, 1000), heads, 2, dim, p, types=types, layers=1, layer=0, seed=9)
    block = c.cache[0, 0, 0].numel() * c.cache.element_size()
    far = (5 << 30) // block
    shape = W.KVShape(1, heads, c.cfg.head_dim, p, far, 1, c.cfg.elem_bytes)
    cache = torch.empty((1, 2, far) + tuple(c.cache.shape[3:]), dtype=c.cache.dtype, device="cuda")
    cache[:, :, far - c.n_blocks:] = c.cache
    table = torch.where(c.table >= 0, c.table + far - c.n_blocks, c.table).cuda()
    lens, starts = c.lens.cuda(), c.starts.cuda()
    dec = D.Decoder(B.make_config(shape), cache.data_ptr(), heads * 2, max_seqs=3, max_blocks=c.max_blocks, x_type=KIND[types[0]],
                    kv_type=KIND[types[1]], max_rows=c.n_rows)
    q = c.queries()
    want, want_lse = c.check(q)
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    assert dec.kv_attend_rows(0, q.cuda(), table, lens, out, starts=starts, lse=lse) == B.KV_OK
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    one = torch.empty((3, heads * 2, dim), dtype=x, device="cuda")
    assert dec.kv_attend(0, q[:3].cuda(), table, lens, one) == B.KV_OK
    ref = A.attend(q[:3].double(), c.values(0), c.values(1), c.table, c.lens, 1 / math.sqrt(dim), c.n_blocks)
    assert ((one.cpu().double() - ref["out"]).abs() <= A.attend_bounds(ref, c.lens, dim, x)[0]).all()
    # new tokens into the last pages
    k, v = (torch.randn((c.n_rows, heads, dim), generator=c.g).to(x).cuda() for _ in range(2))
    norm = D.HeadNorm(None, torch.rand(dim, device="cuda") + 0.5)
    near = D.Decoder(c.cfg, c.cache.data_ptr(), heads * 2, max_seqs=3, max_blocks=c.max_blocks, x_type=KIND[types[0]], kv_type=KIND[types[1]])
    assert dec.kv_put(0, k, v, table, lens, starts=starts, norm=norm) == B.KV_OK
    assert near.kv_put(0, k, v, c.table.cuda(), lens, starts=starts, norm=norm) == B.KV_OK
    assert torch.equal(cache[:, :, far - c.n_blocks:].view(torch.uint8), c.cache.view(torch.uint8))
