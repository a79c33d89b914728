"""Sampling, top logits of few rows and distillation of few rows on the checked build: list pushes, group flags, bins of masses and of
narrowing, and the marks of listed entries are tested against their buffers, and the status word has to stay clean, which the
modules' own fixtures assert."""
import os
import subprocess
import sys

import pytest

from paper_2506_15733_b200 import binding, build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("module,selected", [
    ("test_gpu_rows.py", "sampling or ties or top_logits_match or distillation_matches"),
    ("test_gpu_rows_signed_zero.py", "largest or draws"),
    ("test_gpu_rows_tail.py", "sure_student and f32"),
    ("test_gpu_rows_shares.py", "127990"),
])
def test_row_operators_on_the_checked_build(module, selected):
    if binding.debug_build():
        pytest.skip("already inside the checked build")
    assert os.path.exists(build.LIB_PATH_DEBUG), "build the checked library: python -m paper_2506_15733_b200.build --debug"
    res = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", module), "-m", "gpu", "-x", "-q", "-k",
                          selected], cwd=ROOT, env=dict(os.environ, SPECS_B200_DEBUG="1"), capture_output=True, text=True,
                         timeout=900)
    assert res.returncode == 0 and " passed" in res.stdout, res.stdout[-2000:] + res.stderr[-2000:]
