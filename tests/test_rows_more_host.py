"""What the host code of the decoder's calls hands to kernels, on the CPU."""
import os
import subprocess

import pytest

from tests import launches as L


@pytest.mark.skipif(not os.path.exists(L.HIPCC), reason="needs hipcc")
def test_what_kernels_are_handed(tmp_path):
    obj, exe = str(tmp_path / "host_rows_more.o"), str(tmp_path / "host_rows_more")
    subprocess.run([L.HIPCC, "--offload-host-only", "-x", "hip", "-fPIC", "-std=c++17", "-O1", "-w", "-c",
                    os.path.join(L.ROOT, "tests", "host_rows_more.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", obj, "-o", exe, "-Wl,--unresolved-symbols=ignore-all"], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-1000:] + run.stderr[-3000:]
    assert "host rows more ok" in run.stdout
