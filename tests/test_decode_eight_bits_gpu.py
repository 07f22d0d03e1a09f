"""An 8-bit cache holds the nearest of value / scale: every 16-bit value, over scales where a product with 1 / scale, or a
quotient rounded to 32 bits, comes to lie on the wrong side of the middle between two e4m3 values."""
import pytest
import torch

from paper_2601_20309_amd import binding as B
from paper_2601_20309_amd import decode as D
from paper_2601_20309_amd import workloads as W

pytestmark = pytest.mark.gpu


def nearest(x, scale):
    """e4m3 codes of x / scale: the quotient in 64 bits against the middles of neighbours, ties to the even code.  (x has 11
    digits and fewer, scale 24, a middle 5: a quotient is a middle or 2^-29 of it and more away from one.)"""
    value = torch.arange(0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    middle = (value[1:] + value[:-1]) / 2
    t = x.double().abs() / float(torch.tensor(scale, dtype=torch.float32))
    up, down = torch.bucketize(t, middle, right=True), torch.bucketize(t, middle)      # they differ at a middle
    code = torch.where(up != down, up + (up & 1) * (down - up), up)
    return torch.where(x.isnan(), torch.full_like(code, 0x7F), code) + 128 * torch.signbit(x)


@pytest.mark.parametrize("type_", ["bf16", "fp16"])
@pytest.mark.parametrize("k_scale,v_scale", [(0.02, 0.01), (0.03, 0.0125), (0.7, 0.3), (1.0, 0.1), (448.0, 3e-5)])
def test_every_value_goes_to_its_nearest(type_, k_scale, v_scale):
    x_type = {"bf16": torch.bfloat16, "fp16": torch.float16}[type_]
    shape = W.KVShape(1, 8, 64, 16, 8, 1, 1)
    cache = torch.zeros(shape.cache_dims(), dtype=torch.uint8, device="cuda")
    dec = D.Decoder(B.make_config(shape), cache.data_ptr(), 8, max_seqs=1, max_blocks=8, x_type=getattr(B, f"KV_{type_.upper()}"),
                    kv_type=B.KV_FP8, k_scale=k_scale, v_scale=v_scale)
    x = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(x_type)
    rows = x.view(128, 8, 64).cuda()
    table, lens = torch.arange(8, dtype=torch.int32, device="cuda")[None], torch.tensor([128], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 128], dtype=torch.int32, device="cuda")
    assert dec.kv_put(0, rows, rows, table, lens, starts=starts) == 0
    got = cache.cpu().view(2, -1)
    for which, scale in enumerate((k_scale, v_scale)):
        want = nearest(x.float(), scale)
        nan = x.isnan()
        assert (got[which][nan] & 0x7F == 0x7F).all()
        wrong = (got[which].long() != want)[~nan]
        assert not wrong.any(), f"scale {scale}: {int(wrong.sum())} values are not the nearest, as {x[~nan][wrong][:3].tolist()}"
