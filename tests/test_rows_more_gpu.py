"""Attention of many rows: calls that the documentation allows and that are seldom made."""
import math

import pytest
import torch

from paper_2601_20309_amd import binding as B
from tests import rows_reference as R
from tests.test_rows_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [(3, 0, 5), (70, 0, 200), (0, 0, 0), (1100, 0, 1100)], ids=str)
@pytest.mark.parametrize("before", [1, 37, 300])
def test_rows_before_the_first_request(new, before):
    """They are nobody's, as those behind the last one are."""
    heads = 64 if max(new) > 1000 else 2
    c = Case(new, [n + 60 for n in new], heads, 1, 64, seed=before, behind=before + 4)
    c.check(starts=c.starts + before)
    c.check(starts=c.starts + before, causal=False)


@pytest.mark.parametrize("n", [63, 64, 65, 128, 129])
@pytest.mark.parametrize("new", [1, 20, 80])
def test_requests_around_the_lanes_of_a_wave(n, new):
    lens = [new + (37 * i) % 150 for i in range(n)]
    lens[n - 1], lens[n // 2] = 1500, 0
    Case((new,) * n, lens, 1, 3, 64, seed=n + new).check()


@pytest.mark.parametrize("heads,group", [(1, 1024), (2, 300), (1, 77)])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp8"), ("bf16", "fp4")], ids="-".join)
def test_many_heads_of_a_kv_head(heads, group, types):
    """A row alone has several tiles."""
    Case((1, 2, 0, 3), (200, 33, 5, 700), heads, group, 64, types=types, seed=group).check()
    Case((1,) * 70, (40,) * 70, heads, group, 32, types=types, seed=group).check()


@pytest.mark.parametrize("p", [257, 4000])
def test_pages_longer_than_a_request(p):
    Case((5, 90), (100, 3900), 2, 2, 64, p=p, seed=p).check()


def test_one_query_for_all_rows():
    """A row that is read again and again (rows any distance apart, none among them)."""
    c = Case((40, 5), (300, 90), 2, 2, 64, seed=3)
    q = c.queries()[:1].expand(c.n_rows, -1, -1)
    ref = R.rows(q, c.values(0), c.values(1), c.table, c.lens, c.starts, 1 / math.sqrt(c.dim), True, c.n_blocks)
    one = q[:1].cuda().expand(c.n_rows, -1, -1)
    out = torch.empty(q.shape, dtype=c.x, device="cuda")
    lse = torch.empty(q.shape[:2], device="cuda")
    assert c.dec.kv_attend_rows(c.layer, one, c.table.cuda(), c.lens.cuda(), out, starts=c.starts.cuda(), lse=lse) == B.KV_OK
    c.compare(out, lse, ref)


def test_two_graphs_in_turn():
    """Two recorded calls of one decoder, replayed one after the other: what one leaves behind is nothing to the other."""
    c = Case((3, 250), (9000, 400), 1, 4, 64, seed=19)
    few = torch.tensor([0, 3, 4], dtype=torch.int32)
    q = c.queries()
    qd, table = q.cuda(), c.table.cuda()
    calls, want = [], []
    for starts, lens in ((c.starts, c.lens), (few, torch.tensor([8000, 300], dtype=torch.int32))):
        out, lse = torch.zeros(q.shape, dtype=c.x, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
        s, n = starts.cuda(), lens.cuda()
        call = lambda out=out, lse=lse, s=s, n=n: c.dec.kv_attend_rows(c.layer, qd, table, n, out, starts=s, lse=lse)  # noqa: E731
        assert call() == B.KV_OK
        torch.cuda.synchronize()
        want.append((out.clone(), lse.clone()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            assert call() == B.KV_OK
        calls.append((graph, out, lse, call))       # (call: its tensors have to live as long as the graph)
    for i in (0, 1, 1, 0, 1, 0, 0):
        graph, out, lse = calls[i][:3]
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
