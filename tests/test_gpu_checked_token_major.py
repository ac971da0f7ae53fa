"""The token-major operators on the checked build of the library (-DUBP_DEBUG): the cases of both test files, the row
operators' among them, and damaged plans. A process loads one build, so they run in child processes."""
import os
import re
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2407_19644_b200", "libubp_b200_debug.so")


def child(args):
    if not os.path.exists(LIB):
        from paper_2407_19644_b200 import build
        build.build(debug=True)
    r = subprocess.run([sys.executable] + args, cwd=ROOT, env=dict(os.environ, UBP_B200_LIBRARY=LIB), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    return r.stdout


@pytest.mark.parametrize("files,names,least", [
    (["tests/test_gpu_rows.py", "tests/test_gpu_rows_exact.py"], "test_norm or test_quant_rows or special_values or test_codes", 400),
    (["tests/test_gpu_linear.py", "tests/test_gpu_linear_values.py"], "test_same_result or test_output_alignments or test_kept_blocks or test_fp32", 60)])
def test_cases_run_on_the_checked_build(files, names, least):
    out = child(["-m", "pytest", *files, "-q", "-x", "-m", "gpu", "-k", names])
    assert int(re.search(r"(\d+) passed", out).group(1)) >= least, out[-500:]


def test_damaged_plans_are_noticed():
    out = child([os.path.join("tests", "checked_linear_cases.py")])
    assert "checked linear ok" in out
