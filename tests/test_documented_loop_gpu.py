"""The decode loop that README.md shows, run as it stands there, over an eviction: new tokens stand behind all that
came before them, whatever has left."""
import math
import os
import re

import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W
from tests import decode_reference as R

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def the_loop():
    with open(README) as f:
        text = f.read()
    at = text.index("The model's side of an iteration")
    return compile(re.compile(r"```python\n(.*?)```", re.S).search(text, at).group(1), README, "exec")


def test_tokens_keep_their_places_after_an_eviction():
    shape, prompt, dim = W.KVShape(1, 8, 64, 16, 160, 8), 140 * 16, 64
    g = torch.Generator().manual_seed(3)
    cache = torch.zeros(shape.cache_dims(), dtype=torch.bfloat16, device="cuda")
    eng = B.Engine(B.make_config(shape), cache.data_ptr())
    tab = B.Table(eng, 1)
    inv_freq = (10000.0 ** -(torch.arange(dim // 2, dtype=torch.float64) * 2 / dim)).float().cuda()
    table = torch.full((1, 512), -1, dtype=torch.int32, device="cuda")
    lens, count = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    ids, at = (torch.zeros((1, 512), dtype=torch.int32, device="cuda") for _ in range(2))
    mass = torch.zeros((1, 512), device="cuda")
    position = torch.tensor([[prompt - 1]], dtype=torch.int32, device="cuda")
    make = lambda *n: torch.randn(n, generator=g).to(torch.bfloat16)       # noqa: E731

    def follow():
        b = tab.kv_table_blocks(0)
        table.fill_(-1)
        table[0, :len(b["ids"])] = torch.tensor(b["ids"], dtype=torch.int32, device="cuda")
        lens[0] = b["len"]

    assert tab.kv_table_append(0, prompt)[0] == 0
    follow()
    k, v = make(prompt, 8, dim).cuda(), make(prompt, 8, dim).cuda()
    first = D.Decoder(eng.cfg, cache.data_ptr(), 32, max_seqs=1, max_blocks=512)
    assert first.kv_put(0, k, v, table, lens, starts=torch.tensor([0, prompt], dtype=torch.int32, device="cuda"), rope=D.Rope(inv_freq)) == 0
    left = 0
    for step in range(4):
        assert tab.kv_table_append(0, 1)[0] == 0
        follow()
        position += 1
        k, v, q, out = make(1, 8, dim), make(1, 8, dim), make(1, 32, dim), torch.empty((1, 32, dim), dtype=torch.bfloat16, device="cuda")
        names = dict(eng=eng, cache=cache, inv_freq=inv_freq, tab=tab, table=table, lens=lens, mass=mass, position=position, layer=0,
                     k=k.cuda(), v=v.cuda(), q=q.cuda(), out=out, ids=ids, at=at, count=count, req=0, s=0)
        rows, n = table.clone().cpu(), int(lens[0])
        exec(the_loop(), names)
        torch.cuda.synchronize()
        left += int(count[0])
        # where the token stands: q and its key turned by as many places as there are tokens before it, gone or not
        turn = lambda x: R.turned(x, position.cpu(), inv_freq.cpu(), (dim // 2,), dim, False)   # noqa: E731
        cell = (int(rows[0, (n - 1) // 16]), (n - 1) % 16)
        for got, x in ((names["q"][0], q), (cache[0, 0][cell], k)):
            want = turn(x)[0]
            most = 2.0 ** -8 * want.abs() + 2.0 ** -20 * x.double().abs().max()
            assert ((got.cpu().double() - want).abs() <= most).all(), f"step {step}: not at place {int(position)}"
        assert torch.equal(cache[0, 1][cell].cpu(), v[0])
        ref = R.attend(names["q"].cpu().double(), cache[0, 0].cpu().double(), cache[0, 1].cpu().double(), rows, torch.tensor([n]),
                       1 / math.sqrt(dim), 160)
        bound, _, _ = R.attend_bounds(ref, torch.tensor([n]), dim, torch.bfloat16)
        assert ((out.cpu().double() - ref["out"]).abs() <= bound).all()
        kept = table.clone(), lens.clone()
        follow()
        assert torch.equal(kept[0], table) and torch.equal(kept[1], lens)
    assert left == 13
    tab.kv_table_destroy()
    eng.kv_destroy()
