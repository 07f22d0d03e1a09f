"""The decoder beside torch's differentiation: it has no gradients, and says so."""
import torch
import pytest
import torch.autograd.forward_ad as forward

from paper_2601_20309_amd import binding as B
from tests.test_decode_gpu import Case, rope_of

pytestmark = pytest.mark.gpu


class Calls:
    """Every operator once, each with one of its tensors replaced by name."""

    def __init__(self):
        self.c = c = Case(2, 2, 64, lens=(40, 20), seed=50)
        n, blocks = 2, c.max_blocks
        ints = lambda *d: torch.zeros(d, dtype=torch.int32, device="cuda")      # noqa: E731
        rows = lambda h: torch.randn((n, h, 64), generator=c.g).to(c.x).cuda()  # noqa: E731
        self.t = dict(q=rows(4), out=rows(4), lse=torch.zeros((n, 4), device="cuda"), mass=torch.rand((n, blocks), device="cuda"),
                      mass_out=torch.zeros((n, blocks), device="cuda"), k=rows(2), v=rows(2), q_in=rows(4), q_out=rows(4),
                      table=c.table.cuda(), lens=c.lens.cuda(), ids=ints(n, 2), at=ints(n, 2), count=ints(n),
                      table_out=ints(n, blocks), lens_out=ints(n), weights=torch.rand((n, blocks), device="cuda"),
                      weights_out=torch.zeros((n, blocks), device="cuda"))
        self.rope = rope_of(64)

    def attend(self, **other):
        t = {**self.t, **other}
        return self.c.dec.kv_attend(1, t["q"], t["table"], t["lens"], t["out"], lse=t["lse"], mass=t["mass"], mass_out=t["mass_out"])

    def put(self, **other):
        t = {**self.t, **other}
        return self.c.dec.kv_put(1, t["k"], t["v"], t["table"], t["lens"], q=t["q_in"], q_out=t["q_out"], rope=self.rope)

    def evict(self, **other):
        t = {**self.t, **other}
        return self.c.dec.kv_evict(t["table"], t["lens"], t["weights"], budget=1, n_first=0, n_last=1, evicted_ids=t["ids"],
                                   evicted_at=t["at"], n_evicted=t["count"], table_out=t["table_out"], lens_out=t["lens_out"],
                                   mass_out=t["weights_out"])


def test_tangents_are_refused():
    """A dual tensor's tangent would be dropped without a word; torch.no_grad() does not change that."""
    calls = Calls()
    kept = {k: x.clone() for k, x in calls.t.items()}
    cache = calls.c.cache.clone()
    with forward.dual_level():
        for call, names in ((calls.attend, ("q", "out", "lse", "mass", "mass_out")), (calls.put, ("k", "v", "q_in", "q_out")),
                            (calls.evict, ("weights", "weights_out"))):
            for name in names:
                dual = forward.make_dual(calls.t[name], torch.ones_like(calls.t[name]))
                assert call(**{name: dual}) == B.KV_EINVAL, name
                with torch.no_grad():
                    assert call(**{name: dual}) == B.KV_EINVAL, name
        torch.cuda.synchronize()
        assert torch.equal(calls.c.cache, cache) and all(torch.equal(x, kept[k]) for k, x in calls.t.items())
        # where forward mode is off, and where no tensor carries a tangent, calls go through
        with torch.inference_mode():
            assert calls.attend(q=forward.make_dual(calls.t["q"], torch.ones_like(calls.t["q"]))) == B.KV_OK
        assert calls.attend() == B.KV_OK and calls.put() == B.KV_OK and calls.evict() == B.KV_OK


def test_transforms_are_refused():
    """Inside torch.func's transforms tensors stand for others: none of these calls can be differentiated or batched."""
    calls = Calls()
    before = calls.t["out"].clone()
    codes = []

    def f(q):
        codes.append(calls.attend(q=q))
        return q.float().sum()

    q = calls.t["q"]
    torch.func.jvp(f, (q,), (torch.ones_like(q),))
    torch.func.grad(f)(q)
    torch.func.vmap(f)(q.expand(3, -1, -1, -1))
    torch.cuda.synchronize()
    assert codes == [B.KV_EINVAL] * 3 and torch.equal(calls.t["out"], before)


def test_what_is_written_has_another_version():
    """Outputs count as changed in place, inputs do not; a call that is refused changes nothing."""
    calls = Calls()
    t, versions = calls.t, lambda: {k: x._version for k, x in calls.t.items()}     # noqa: E731
    for call, outputs in ((calls.attend, {"out", "lse", "mass_out"}), (calls.put, {"q_out"}),
                          (calls.evict, {"ids", "at", "count", "table_out", "lens_out", "weights_out"})):
        before = versions()
        assert call() == B.KV_OK
        assert {k for k, n in versions().items() if n != before[k]} == outputs
    # in place
    before = versions()
    assert calls.attend(mass_out=None, out=t["q"]) == B.KV_OK and calls.put(q_out=t["q_in"]) == B.KV_OK
    assert calls.evict(table_out=None, lens_out=None, weights_out=None) == B.KV_OK
    assert {k for k, n in versions().items() if n != before[k]} == {"lse", "mass", "q", "q_in", "ids", "at", "count", "table", "lens", "weights"}
    before = versions()
    assert calls.attend(lens=t["lens"].long()) == B.KV_EINVAL and calls.evict(table=t["table"].long()) == B.KV_EINVAL
    assert calls.put(q_out=None) == B.KV_EINVAL and versions() == before


def test_a_backward_pass_sees_that_what_it_saved_was_overwritten():
    """The same out for one layer after the other: a product that saved the first one's cannot go backward."""
    calls = Calls()
    w = torch.ones((), device="cuda", requires_grad=True)
    assert calls.attend() == B.KV_OK
    y = (w * calls.t["out"].float()).sum() + (w * calls.t["lse"]).sum()
    y.backward()                                # nothing has been overwritten
    y = (w * calls.t["lse"]).sum()
    assert calls.attend() == B.KV_OK
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_inference_tensors_are_written():
    calls = Calls()
    with torch.inference_mode():
        out = torch.zeros_like(calls.t["out"])
        assert calls.attend(out=out) == B.KV_OK
    again = torch.zeros_like(out)
    assert calls.attend(out=again) == B.KV_OK and torch.equal(out, again)
    assert calls.attend(out=out) == B.KV_OK and torch.equal(out, again)
