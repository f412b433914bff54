"""The batch experts' operators under the bounds-checked build of the library (``-DDX_CHECKED``): ragged groups, rows in place and
gathered, written in order and scattered, outside every group, long contractions; the loss of ragged rows in pieces and in one.
What their kernels place by data -- offsets, sorted rows, the list of rows that count, halves of tiles, pieces of dz -- is checked
against its buffers; a violated bound is recorded in the device status word and the access skipped.  Every one of these tests
asserts that the status word stayed clean."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("source", ["dx_mm.cuh", "dx_experts_mm.cu", "dx_head.cu"])
def test_kernels_that_index_by_data_have_bounds_checks(source):
    with open(os.path.join(ROOT, "paper_2607_24434_b200", "csrc", source)) as f:
        assert f.read().count("DX_BOUNDS(") >= 5


@pytest.mark.gpu
def test_batch_experts_under_the_checked_build():
    from paper_2607_24434_b200 import build as dx_build
    lib = dx_build.build(checked=True)
    env = dict(os.environ, DX_LIB_PATH=lib)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider",
           *(os.path.join(ROOT, "tests", name) for name in ("test_gpu_experts_batch.py", "test_gpu_experts_batch_edges.py",
                                                            "test_gpu_head_loss.py", "test_gpu_head_loss_edges.py")),
           "-k", "grouped_products or groups_matrices or forward_and_backward or combination or bad_rows or nothing_to_do or one_after "
                 "or without_a_row or in_order or exact or very_long or loss_and_gradients or workspace or none_of_which or kept_and "
                 "or short_last or listed_by or weight_zero or graphs"]
    res = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    tail = (res.stdout + res.stderr)[-3000:]
    assert res.returncode == 0, tail
    assert " passed" in res.stdout and "failed" not in res.stdout, tail
