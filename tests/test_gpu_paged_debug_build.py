"""The tests of the paged cache's calls under the checked build of the library (-DPLORA_DEBUG): every unit, partial result,
output row and block-table column that the plan and the attention kernels use is compared with its bounds, and one outside
would show as PLORA_ERR_DEBUG_CHECK in the status word, which the tests look at after each call."""
import os
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

ROOT = Path(__file__).resolve().parent.parent


def test_paged_cases_pass_under_the_checked_build():
    env = dict(os.environ, PLORA_DEBUG_BUILD="1")
    run = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_paged.py", "tests/test_gpu_paged_edges.py", "-x", "-q", "-m", "gpu",
                          "-p", "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    assert run.returncode == 0, run.stdout[-3000:] + run.stderr[-1000:]
    assert " passed" in run.stdout and "failed" not in run.stdout
