"""What the compiler makes of attention of many rows, without a GPU."""
import os
import re
import subprocess

import pytest

from paper_2601_20309_amd import build
from tests import launches as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.HIPCC), reason="needs hipcc")


def compiled(tmp_path, kernels, *flags):
    """The assembly of these kernels, and what the compiler had to say."""
    src, out = tmp_path / "kernels.hip", str(tmp_path / "kernels.s")
    src.write_text('#include <hip/hip_runtime.h>\n#include "kv_rows_kernels.hpp"\nnamespace dkv {\n'
                   + "".join(f"template __global__ void {k}(const RowsParams);\n" for k in kernels) + "}\n")
    run = subprocess.run([L.HIPCC, *build.HIPCC_FLAGS, *flags, "-I", build.CSRC, "--cuda-device-only", "-S", str(src), "-o", out],
                         capture_output=True, text=True, check=True, timeout=600)
    with open(out) as f:
        return f.read(), [line for line in run.stderr.splitlines() if "packed-fp32-ops" not in line]


def test_m0_is_the_direct_loads_alone(tmp_path):
    """They set it in assembly, and say so; nothing that the compiler makes has a value of its own there."""
    with open(os.path.join(build.CSRC, "kv_rows_kernels.hpp")) as f:
        blocks = re.findall(r"asm volatile\((.*?)\);", f.read(), re.S)
    assert [b for b in blocks if "m0" in b.split(":")[0]] and all('"m0"' in b.split(":")[-1] for b in blocks if "m0" in b.split(":")[0])
    text, said = compiled(tmp_path, ["kv_rows_kernel<Bf16, kBits16, 64, 128>", "kv_rows_kernel<Fp16, kBits16, 64, 32>"])
    assert not [line for line in said if "warning" in line and "unused" not in line]
    ours = "".join(re.findall(r";;?#ASMSTART(.*?);;?#ASMEND", text, re.S))
    assert len(re.findall(r"\bm0\b", ours)) == len(re.findall(r"\bm0\b", text)) > 0


def test_no_kernel_keeps_what_it_needs_in_scratch_memory(tmp_path):
    """Heads of 256 dimensions, which take most registers; and no bound that the compiler cannot keep."""
    kernels = [f"kv_rows_kernel<{x}, {kind}, 256, {rows}>" for x, kind in (("Bf16", "kBits16"), ("Bf16", "kBits8"), ("Fp16", "kBits4")) for rows in (32, 128)]
    kernels += ["kv_rows_kernel<Fp16, kBits16, 128, 32>", "kv_rows_kernel<Bf16, kBits8, 192, 32>"]
    text, said = compiled(tmp_path, kernels)
    sizes = [int(n) for n in re.findall(r"\.private_segment_fixed_size:\s*(\d+)", text)]
    assert sizes == [0] * len(kernels)
    assert not [line for line in said if "warning" in line and "unused" not in line], said
