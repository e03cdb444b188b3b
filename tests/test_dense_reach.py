"""The tile of every product of the dense operators reaches its operands with 32-bit offsets,
over all sizes (tests/sanitize/dense_reach.cpp, host code: no GPU is needed)."""
import os
import subprocess

import pytest

from paper_2608_09388_amd import binding as shc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
HIPCC = os.path.join(ROCM, "bin", "hipcc")


def test_offsets_of_the_chosen_tiles(tmp_path):
    source = os.path.join(ROOT, "tests", "sanitize", "dense_reach.cpp")
    if not os.path.exists(HIPCC) or not os.path.exists(source):
        pytest.skip("hipcc or the program's source not found")
    shc.load()
    exe = str(tmp_path / "reach")
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-O1",
                    "-std=c++17", "-I", os.path.join(ROOT, "include"), source, "-x", "none",
                    shc.LIB_PATH, "-Wl,-rpath," + os.path.dirname(shc.LIB_PATH), "-o", exe],
                   check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "bad 0" in r.stdout, r.stdout + r.stderr
    assert int(r.stdout.split()[-3]) > 4000, r.stdout
