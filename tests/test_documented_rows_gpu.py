"""The calls for prompts that README.md shows, run as they stand there, and in 4 bits as it says."""
import math
import os
import re

import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import decode_reference as A
from tests import rows_reference as R

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def the_calls():
    with open(README) as f:
        text = f.read()
    at = text.index("Prompts, parts of them, drafted tokens")
    return compile(re.compile(r"```python\n(.*?)```", re.S).search(text, at).group(1), README, "exec")


def test_prompts_as_documented():
    dim, new, lens = 128, (70, 3), (70, 40)
    shape = W.KVShape(1, 8, dim, 16, 24, 8)
    g = torch.Generator().manual_seed(1)
    cache = torch.randn(shape.cache_dims(), generator=g).to(torch.bfloat16).cuda()
    eng = B.Engine(B.make_config(shape), cache.data_ptr())
    table = torch.full((2, 512), -1, dtype=torch.int32)
    table[0, :5], table[1, :3] = torch.arange(5, dtype=torch.int32), torch.arange(9, 12, dtype=torch.int32)
    inv_freq = 10000.0 ** -(torch.arange(dim // 2).float() / (dim // 2))
    draw = lambda h: torch.randn((73, h, dim), generator=g).to(torch.bfloat16)  # noqa: E731
    q, k, v, weights = draw(32), draw(8), draw(8), [torch.rand(dim, generator=g) + 0.5 for _ in range(2)]
    length, starts = torch.tensor(lens, dtype=torch.int32), torch.tensor([0, 70, 73], dtype=torch.int32)
    names = dict(D=D, eng=eng, cache=cache, q_weight=weights[0].cuda(), k_weight=weights[1].cuda(), rope=D.Rope(inv_freq.cuda()), layer=0,
                 k=k.cuda(), v=v.cuda(), q=q.cuda(), out=torch.empty_like(q, device="cuda"), table=table.cuda(), lens=length.cuda(),
                 starts=starts.cuda())
    exec(the_calls(), names)
    torch.cuda.synchronize()
    place = torch.cat([torch.arange(70), torch.arange(37, 40)])[None]
    want = A.turned(R.normed(q, weights[0], 1e-6), place, inv_freq, (dim // 2,), dim, False)
    got = names["q"].cpu().double()
    # angles and norms in 32 bits, rounded to bf16
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -17 * want.abs().max()).all()
    ref = R.rows(names["q"].cpu(), cache[0, 0].cpu().double(), cache[0, 1].cpu().double(), table, length, starts, 1 / math.sqrt(dim), True, 24)
    bound, _ = R.rows_bounds(ref, dim, torch.bfloat16)
    assert ((names["out"].cpu().double() - ref["out"]).abs() <= bound).all()
    eng.kv_destroy()


def test_a_cache_in_4_bits_is_rotated_as_any_other():
    """Blocks of a 4-bit cache go out and come back, and attention over them is what it was."""
    heads, dim, p, blocks = 2, 128, 16, 12
    shape = W.KVShape(2, heads, D.fp4_head_bytes(dim), p, blocks, 8, elem_bytes=1)
    cache = torch.zeros(shape.cache_dims(), dtype=torch.uint8, device="cuda")
    eng = B.Engine(B.make_config(shape), cache.data_ptr())
    dec = D.Decoder(eng.cfg, cache.data_ptr(), 4, max_seqs=1, max_blocks=4, kv_type=B.KV_FP4, max_rows=60)
    g = torch.Generator(device="cuda").manual_seed(2)
    draw = lambda h: torch.empty((60, h, dim), dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    q, k, v = draw(4), draw(heads), draw(heads)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, lens, starts = ints([5, 2, 7, 0]), ints(60), ints(0, 60)
    before, after = torch.empty_like(q), torch.empty_like(q)
    assert dec.kv_put(1, k, v, table, lens, starts=starts) == B.KV_OK
    assert dec.kv_attend_rows(1, q, table, lens, before, starts=starts) == B.KV_OK
    torch.cuda.synchronize()
    assert eng.kv_swap_out([5, 2, 7, 0], [3, 1, 0, 6]) == B.KV_OK and eng.kv_wait() == B.KV_OK
    cache.fill_(255)
    torch.cuda.synchronize()
    assert eng.kv_swap_in([3, 1, 0, 6], [10, 11, 1, 4]) == B.KV_OK and eng.kv_wait() == B.KV_OK
    assert dec.kv_attend_rows(1, q, ints([10, 11, 1, 4]), lens, after, starts=starts) == B.KV_OK
    assert torch.equal(before, after)
    eng.kv_destroy()
