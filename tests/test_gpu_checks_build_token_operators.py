"""The bounds-check build (libarb_checks.so, -DARB_CHECKS) under the operators around a token: the tests of arb_rope_append*, arb_attn_rules
and arb_logits run once more in a child process that loads it, as test_gpu_checks_build.py does for the kernels they stand on."""
import os
import re
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent

FILES = ["tests/test_gpu_rope.py", "tests/test_gpu_rules.py", "tests/test_gpu_rules_edges.py", "tests/test_gpu_logits.py"]


@pytest.mark.parametrize("file", FILES)
def test_token_operators_under_the_bounds_check_build(file):
    from paper_2512_05033_b200 import build
    build.build(checks=True)
    # without the cases that time a call
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-s", "-m", "gpu", "-k", "not long_lists", file],
                       cwd=ROOT, env=dict(os.environ, ARB_LIB_VARIANT="checks"), capture_output=True, text=True, timeout=900)
    tail = r.stdout[-3000:] + r.stderr[-2000:]
    assert r.returncode == 0, tail
    m = re.search(r"guard zones: (\d+) bytes checked, (\d+) overwritten", r.stdout)
    assert m is not None and int(m.group(1)) > 0 and int(m.group(2)) == 0, tail
