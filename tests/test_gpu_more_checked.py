"""The 8-bit floating-point projection, norm and rotation with their gradients, and the bookkeeping of pages on the checked build
(libjab_checked.so): the tests' values, and no check that fires."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("file,which", [
    ("test_gpu_fp8.py", "(linear and (1-6144 or 65-2560 or 129-257 or 3001-6144)) or pitches or serves_a_fitted or quantize_bit"),
    ("test_gpu_norm_rope.py", "(forward and (37-4 or 1001 or 5-0)) or in_place or (write and (333 or 64-32)) or (backward and (37-4 or 130-96)) or no_tokens"),
    ("test_gpu_plan.py", "release or page_numbers or steps")])
def test_no_check_fires(file, which):
    from paper_2609_34866_gb300 import build
    build.build(checked=True)
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", os.path.join("tests", file), "-k", which],
                       cwd=ROOT, env=dict(os.environ, JAB_CHECKED="1"), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "passed" in r.stdout, r.stdout[-3000:] + r.stderr[-3000:]
