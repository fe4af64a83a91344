"""The small cases of the norm's, the checkpoints' and the attention's GPU tests on the CPU, kernels run lane by lane (tests/lanes)."""
import os
import subprocess
import sys

import pytest

TESTS = os.path.dirname(os.path.abspath(__file__))
LANES = os.path.join(TESTS, "lanes")
sys.path.insert(0, LANES)
import lanes_build  # noqa: E402


@pytest.fixture(scope="session")
def lanes(tmp_path_factory):
    return lanes_build.build(str(tmp_path_factory.mktemp("lanes")))


RUNS = [
    # order of wavefronts and blocks (1: descending); file; selection
    (1, "test_gpu_norm.py", "not graph and not many_rows and not turns and not larger and not 16383 and not 8200 and not 4099 and not 2500"),
    (0, "test_gpu_norm.py", "channels and (257 or 65 or 2056) or checkpoint and 100"),
    (1, "test_gpu_relattn.py", "not larger and not graph and not many"),
    (0, "test_gpu_relattn.py", "test_attention and (m2_h4 or d96 or d9_)"),
    (0, "test_gpu_relattn.py", "many_blocks and 50-1 and (33 or 40 or 128)"),
    (1, "test_gpu_operators.py", "test_block or differences or scales"),
]


@pytest.mark.parametrize("late,name,select", RUNS, ids=["%s-%s" % (r[1][9:-3], "late" if r[0] else "early") for r in RUNS])
def test_gpu_tests_on_lanes(lanes, late, name, select):
    env = dict(os.environ, LPM_LANES=lanes, LPM_LANES_LATE=str(late), PYTHONPATH=os.pathsep.join([LANES, os.environ.get("PYTHONPATH", "")]))
    cmd = [sys.executable, "-m", "pytest", "-p", "lanes_plugin", "-p", "no:cacheprovider", "-q", "-m", "gpu", os.path.join(TESTS, name), "-k", select]
    r = subprocess.run(cmd, env=env, cwd=os.path.dirname(TESTS), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-6000:] + r.stderr[-3000:]
    assert " passed" in r.stdout and " failed" not in r.stdout
