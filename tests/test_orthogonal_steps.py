"""The powers of two that Newton-Schulz operands are held times, which the host takes from the polynomials (no GPU):
tests/orthogonal_steps_main.cpp, compiled with the host's part of csrc/orthogonal.hip alone."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")), reason="hipcc not found")
def test_ranges_of_operands(tmp_path):
    exe = str(tmp_path / "orthogonal_steps")
    # (the kernels' code object stays undefined: nothing is launched)
    subprocess.run([HIPCC if os.path.exists(HIPCC) else "hipcc", "-O2", "-std=c++17", "--offload-arch=gfx950", "--cuda-host-only", "-x", "hip",
                    "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "orthogonal_steps_main.cpp"),
                    "-Wl,--unresolved-symbols=ignore-all", "-o", exe], check=True, stdout=subprocess.PIPE, stderr=subprocess.PIPE)
    out = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr
