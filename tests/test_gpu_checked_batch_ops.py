"""The batch operators under the bounds-checked build of the library (``-DDX_CHECKED``): the small ragged shapes, the
masks, ties and odd lists, and rows that follow one another, whose kernels index by data -- ids, marks, hash places, runs and
candidate lists, histograms, the permutation.  A violated bound is recorded in the device status word and the access
skipped; every one of these tests asserts that the status word stayed clean."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("source", ["dx_batch_route.cu", "dx_logprobs.cu", "dx_distill.cu"])
def test_kernels_that_index_by_data_have_bounds_checks(source):
    with open(os.path.join(ROOT, "paper_2607_24434_b200", "csrc", source)) as f:
        assert f.read().count("DX_BOUNDS(") >= 5


@pytest.mark.gpu
def test_batch_operators_under_the_checked_build():
    from paper_2607_24434_b200 import build as dx_build
    lib = dx_build.build(checked=True)
    env = dict(os.environ, DX_LIB_PATH=lib)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider",
           os.path.join(ROOT, "tests", "test_gpu_batch_ops.py"), os.path.join(ROOT, "tests", "test_gpu_batch_edges.py"),
           "-k", "small_and_ragged or ties or masks or masked or odd_lists or bad_ or put_aside or nearly_equal or far_from "
                 "or route_grad or follow_one_another or longest_rows or whole_vocabulary or lists_outside"]
    res = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    tail = (res.stdout + res.stderr)[-3000:]
    assert res.returncode == 0, tail
    assert " passed" in res.stdout and "failed" not in res.stdout, tail
