"""Host code of attention of many rows, of a cache in 4 bits and of normed heads on the CPU: what is refused, what is
launched, and where it may write; and the reference's own arithmetic."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

from paper_2601_20309_amd import binding as B
from tests import launches as L
from tests import rows_reference as R

ROOT = L.ROOT


@pytest.mark.skipif(not os.path.exists(L.HIPCC), reason="needs hipcc")
def test_rows_host_code(tmp_path):
    obj, exe = str(tmp_path / "host_rows.o"), str(tmp_path / "host_rows")
    subprocess.run([L.HIPCC, "--offload-host-only", "-x", "hip", "-fPIC", "-std=c++17", "-O1", "-w", "-c",
                    os.path.join(ROOT, "tests", "host_rows.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", obj, "-o", exe, "-Wl,--unresolved-symbols=ignore-all"], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-1000:] + run.stderr[-3000:]
    assert "host rows ok" in run.stdout


def test_arguments_are_laid_out_as_the_header_says(tmp_path):
    src, exe = tmp_path / "sizes.c", str(tmp_path / "sizes")
    structs = {B.kv_decoder_config: ("kv_decoder_config", "max_rows"), B.kv_put_args: ("kv_put_args", "norm_eps"),
               B.kv_attend_rows_args: ("kv_attend_rows_args", "lse")}
    lines = "".join(f'printf("%zu %zu\\n", sizeof({n}), offsetof({n}, {m}));' for n, m in structs.values())
    src.write_text(f'#include <stddef.h>\n#include <stdio.h>\n#include "duplexkv.h"\nint main(void) {{ {lines} return KV_FP4 != {B.KV_FP4}; }}\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    for i, (struct, (_, member)) in enumerate(structs.items()):
        assert (C.sizeof(struct), getattr(struct, member).offset) == (int(out[2 * i]), int(out[2 * i + 1])), struct


def test_calls_without_a_handle():
    assert B.lib.kv_attend_rows(None, C.byref(B.kv_attend_rows_args()), None) == B.KV_EINVAL


def test_the_reference_in_4_bits():
    """What the reference writes it reads back: numbers there are as they were, others to the nearest."""
    for dtype, (lo, hi) in R.POWERS.items():
        x = torch.cat([R.NUMBERS, -R.NUMBERS]).repeat(2).view(1, 1, 32)
        for e in (lo, -3, 0, hi):
            rows = R.fp4_rows(x * 2.0 ** e, dtype)
            assert rows.shape == (1, 17) and rows[0, 16] == e + 127
            assert torch.equal(R.fp4_values(rows, 1, 32), x * 2.0 ** e)
    y = torch.randn((50, 3, 64), generator=torch.Generator().manual_seed(1)).double()
    back = R.fp4_values(R.fp4_rows(y, torch.bfloat16), 3, 64)
    power = torch.exp2(torch.floor(torch.log2(y.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True))) - 2)
    off = ((back - y).unflatten(-1, (-1, 32)).abs() / power)
    assert off.max() <= 2.0 and (off <= 1.0)[(y.unflatten(-1, (-1, 32)).abs() / power) <= 7].all()


def test_the_reference_of_rows():
    """Against a softmax written out, rows that see nothing and rows of nobody among them."""
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(n, generator=g).double() for n in ((5, 2, 4), (3, 4, 1, 4), (3, 4, 1, 4)))
    table, lens, starts = torch.tensor([[2, 0], [-1, 1]]), torch.tensor([2, 6]), torch.tensor([0, 3, 4])
    ref = R.rows(q, k, v, table, lens, starts, 0.5, True, 3)
    assert (ref["out"][0] == 0).all() and ref["lse"][0].eq(-math.inf).all() and ref["out"][4].isnan().all()
    assert torch.allclose(ref["out"][1], v[2, 0].expand(2, 4)) and torch.allclose(ref["out"][2, 1], torch.softmax(k[2, :2, 0] @ q[2, 1] * 0.5, 0) @ v[2, :2, 0])
    assert torch.allclose(ref["out"][3, 0], torch.softmax(k[1, :2, 0] @ q[3, 0] * 0.5, 0) @ v[1, :2, 0])
