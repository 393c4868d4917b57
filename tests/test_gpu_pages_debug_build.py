"""The paged 8-bit store and its attention on the bounds-checking build: a guarded store that misses sets bad_index, which every
test that counts its status would see."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pages_on_the_bounds_checking_build():
    from paper_2602_10825_b200 import build as fc_build
    fc_build.build(debug_bounds=True)
    run = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_gpu_pages.py", "-m", "gpu", "-k",
                          "append or long_life or over_pages or of_a_span or strides or rolling"],
                         cwd=ROOT, env={**os.environ, "FC_LIB": "debug"}, capture_output=True, text=True, timeout=600)
    assert run.returncode == 0, run.stdout[-3000:] + run.stderr[-2000:]
