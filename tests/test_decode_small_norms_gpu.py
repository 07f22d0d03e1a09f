"""Norms of heads whose squares are too small for 32 bits, with an eps that does not hide them."""
import pytest
import torch

from tests.test_decode_fp4_gpu import Put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -140, 2.0 ** -100])
@pytest.mark.parametrize("x,kv,powers", [("bf16", "bf16", (-40, -44, -50, -60, -62, -63, -64, -70, -76, -100, -125)), ("bf16", "fp8", (-64, -80, 0)),
                                         ("bf16", "fp4", (-63, -64, -100)), ("fp16", "fp16", (-12, -23))])
@pytest.mark.parametrize("heads,dim,rot,interleaved", [(2, 64, 64, False), (3, 96, 48, True), (2, 128, 128, False), (2, 256, 256, False),
                                                       (5, 40, 0, False)])
def test_small_heads(eps, x, kv, powers, heads, dim, rot, interleaved):
    """Each token's heads are 2^power times as much, every third head 2^20 times that."""
    if kv == "fp4" and dim % 32:
        pytest.skip("heads in 4 bits have a multiple of 32 dimensions")
    c = Put((len(powers),), (9,), heads, 2, dim, x=x, kv=kv, rot=rot, interleaved=interleaved, seed=dim, eps=eps,
            k_scale=0.02 if kv == "fp8" else 1.0)
    up = torch.exp2(torch.tensor(powers).float())[:, None, None]
    for name in ("q", "k"):
        t = getattr(c, name)
        t[:] = (t.float() * up).to(c.x)
        t[:, 2::3] = (t[:, 2::3].float() * (2.0 ** 20 if x == "bf16" else 1.0)).to(c.x)
        t[t == 0] = up.expand(t.shape).to(c.x)[t == 0]         # (no head of zeros alone)
    c.check()


def test_heads_of_zeros():
    """With an eps they stay what they are; 0 / 0 without."""
    for eps in (1e-6, 2.0 ** -100, 0.0):
        c = Put((3,), (0,), 2, 2, 64, rot=0, seed=1, eps=eps)
        c.q[1], c.k[1] = 0, 0
        c.run()
        got = c.cache[c.layer, 0, int(c.table[0, 0])].cpu()
        assert (c.q_out[1].isnan().all() and got[1].isnan().all()) if eps == 0 else ((c.q_out[1] == 0).all() and (got[1] == 0).all())
        assert torch.isfinite(c.q_out[::2]).all() and torch.isfinite(got[:3:2]).all()
