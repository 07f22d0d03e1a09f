"""The decoder's host code and kv_table_drop on the CPU: what is refused, what is launched, where it
may write, bad pages, and the order of weights."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2601_20309_amd import binding as B
from tests import launches as L

ROOT = L.ROOT


@pytest.mark.skipif(not os.path.exists(L.HIPCC), reason="needs hipcc")
def test_decoder_host_code(tmp_path):
    obj, exe = str(tmp_path / "host_decode.o"), str(tmp_path / "host_decode")
    subprocess.run([L.HIPCC, "--offload-host-only", "-x", "hip", "-fPIC", "-std=c++17", "-O1", "-w", "-c",
                    os.path.join(ROOT, "tests", "host_decode.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", obj, "-o", exe, "-Wl,--unresolved-symbols=ignore-all"], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-1000:] + run.stderr[-3000:]
    assert "host decode ok" in run.stdout


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_blocks_leave_a_request(tmp_path):
    exe = str(tmp_path / "host_drop")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "host_drop.cpp"),
                    os.path.join(ROOT, "paper_2601_20309_amd", "csrc", "kv_table.cpp"), "-static-libasan", "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-1000:] + run.stderr[-3000:]
    assert "host drop ok" in run.stdout


def test_arguments_are_laid_out_as_the_header_says(tmp_path):
    """Sizes and last members of the argument structures, C against ctypes."""
    src, exe = tmp_path / "sizes.c", str(tmp_path / "sizes")
    structs = {B.kv_decoder_config: ("kv_decoder_config", "weigh"), B.kv_rows: ("kv_rows", "head"),
               B.kv_put_args: ("kv_put_args", "position_stride"), B.kv_attend_args: ("kv_attend_args", "mass_stride"),
               B.kv_evict_args: ("kv_evict_args", "n_evicted")}
    lines = "".join(f'printf("%zu %zu\\n", sizeof({n}), offsetof({n}, {m}));' for n, m in structs.values())
    src.write_text(f'#include <stdio.h>\n#include "duplexkv.h"\nint main(void) {{ {lines} return 0; }}\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    for i, (struct, (_, member)) in enumerate(structs.items()):
        assert (C.sizeof(struct), getattr(struct, member).offset) == (int(out[2 * i]), int(out[2 * i + 1])), struct


def test_calls_without_a_handle():
    assert B.lib.kv_decoder_create(None, None, None, None) == B.KV_EINVAL
    assert B.lib.kv_decoder_destroy(None) == B.KV_EINVAL
    for call, args in ((B.lib.kv_put, B.kv_put_args()), (B.lib.kv_attend, B.kv_attend_args()), (B.lib.kv_evict, B.kv_evict_args())):
        assert call(None, C.byref(args), None) == B.KV_EINVAL
    assert B.lib.kv_table_drop(None, 0, None, 0) == B.KV_EINVAL
