"""What goes into an 8-bit cache, on the CPU: value / scale as the kernel takes it, for every 16-bit value."""
import os
import subprocess

import pytest

from tests import launches as L


@pytest.mark.skipif(not os.path.exists(L.HIPCC), reason="needs hipcc")
def test_values_over_scales(tmp_path):
    obj, exe = str(tmp_path / "host_scale.o"), str(tmp_path / "host_scale")
    subprocess.run([L.HIPCC, "--offload-host-only", "-x", "hip", "-fPIC", "-std=c++17", "-O2", "-mfma", "-w", "-c",
                    os.path.join(L.ROOT, "tests", "host_scale.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", obj, "-o", exe, "-Wl,--unresolved-symbols=ignore-all"], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-1000:] + run.stderr[-3000:]
    assert "host scale ok" in run.stdout
