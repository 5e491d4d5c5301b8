"""The kernels with hand-placed loads, as they are compiled for gated products, against the checking build (ordinary loads with
compiler-placed waits): bit for bit, as test_gpu_plain_loads.py has it for the products alone."""
import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_hand_placed_loads_agree_with_ordinary_loads(tmp_path):
    from paper_2007_13055_amd import build as hip_build
    import gated_plain_loads_cases as cases
    assert os.path.exists(hip_build.LIB_PLAIN), "the checking build is missing: python -m paper_2007_13055_amd.build"
    mine = cases.run_cases()
    out = tmp_path / "plain.npz"
    r = subprocess.run([sys.executable, "-u", os.path.join(ROOT, "tests", "gated_plain_loads_cases.py"), hip_build.LIB_PLAIN, str(out)],
                       capture_output=True, text=True, timeout=110, cwd=ROOT)
    assert r.returncode == 0, r.stdout + r.stderr
    assert os.path.abspath(hip_build.LIB_PLAIN) in r.stdout
    plain = np.load(out)
    assert sorted(plain.files) == sorted(mine)
    for name in mine:
        assert np.all(np.isfinite(mine[name])) and np.array_equal(mine[name], plain[name]), f"{name}: the two builds differ"
