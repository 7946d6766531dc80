"""The tests of plain tables and of rows in 8 bits on the index-check build of the library (see test_gpu_debug_build.py): every test
must pass as usual and leave the debug word at zero."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_tables_and_rows_in_8_bits_run_clean_on_the_index_check_build():
    if os.environ.get("ROBE_LIBRARY"):
        pytest.skip("already inside the child run")
    from paper_2108_02191_b200 import build
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_table.py", "tests/test_gpu_rows8.py", "-m", "gpu", "-x", "-q"],
                       env=dict(os.environ, ROBE_LIBRARY=build.build_debug()), cwd=ROOT, capture_output=True, text=True, timeout=3000)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
    assert " passed" in r.stdout


def test_plans_of_the_attention_run_clean_on_the_index_check_build():
    if os.environ.get("ROBE_LIBRARY"):
        pytest.skip("already inside the child run")
    from paper_2108_02191_b200 import build
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_attend_plans.py", "-m", "gpu", "-x", "-q"],
                       env=dict(os.environ, ROBE_LIBRARY=build.build_debug()), cwd=ROOT, capture_output=True, text=True, timeout=3000)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
    assert " passed" in r.stdout
