"""Work lists of the matrix products (GemmGrid::item over the planners' grids), walked on the host by work_lists_harness.hip.  Host code only: no GPU."""
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parents[1]
HIPCC = shutil.which("hipcc") or shutil.which("/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    if HIPCC is None:
        pytest.skip("needs hipcc")
    exe = tmp_path_factory.mktemp("work_lists") / "harness"
    build = subprocess.run([HIPCC, "--offload-host-only", "-std=c++17", "-O2", f"-I{ROOT / 'include'}", f"-I{ROOT / 'paper_2503_17924_amd' / 'csrc'}",
                            str(ROOT / "tests" / "work_lists_harness.hip"), "-o", str(exe)], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    return exe


def test_every_tile_and_part_once(harness):
    run = subprocess.run([str(harness)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, (run.stdout + run.stderr)[-4000:]
    assert "work lists: ok" in run.stdout


def test_plan_of_the_largest_calls_is_short(harness):
    """A call's host time does not grow with its tiles."""
    run = subprocess.run([str(harness), "largest"], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout + run.stderr
