"""The decoder's limits, on the CPU: what it refuses because no launch or 32-bit number holds it."""
import os
import subprocess

import pytest

from tests import launches as L


@pytest.fixture(scope="module")
def limits(tmp_path_factory):
    if not os.path.exists(L.HIPCC):
        pytest.skip("needs hipcc")
    at = tmp_path_factory.mktemp("limits")
    obj, exe = str(at / "host_decode_limits.o"), str(at / "host_decode_limits")
    subprocess.run([L.HIPCC, "--offload-host-only", "-x", "hip", "-fPIC", "-std=c++17", "-O1", "-w", "-c",
                    os.path.join(L.ROOT, "tests", "host_decode_limits.cpp"), "-o", obj], check=True)
    subprocess.run(["g++", obj, "-o", exe, "-Wl,--unresolved-symbols=ignore-all"], check=True)
    return exe


@pytest.mark.parametrize("what", ["scales", "grids"])
def test_limits(limits, what):
    run = subprocess.run([limits, what], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-1000:] + run.stderr[-3000:]
    assert "host decode limits ok" in run.stdout
