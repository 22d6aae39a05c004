"""Layer norm and the 8-bit entry points under the debug-bounds build (every global address a kernel computes checked against the buffers of its call): all of
their tests but those of very large tensors, of the choice of forms and of captured graphs (the table of buffers is copied from the host for
each call, and a captured copy reads the table of the last call set up), in a child process, because a process loads one library."""
import os
import subprocess
import sys

import pytest
from conftest import ROOT

pytestmark = pytest.mark.gpu
FILES = ["test_layer_norm_gpu.py", "test_layer_norm_far_rows_gpu.py", "test_blocks8_gpu.py", "test_blocks8_zeros_gpu.py", "test_layer8_gpu.py",
         "test_matmul8_gpu.py", "test_matmul8_scales_gpu.py", "test_matmul8_waits_gpu.py"]


def test_layer_norm_and_8_bit_tests_pass_under_the_debug_bounds_build():
    from paper_2110_15032_b200.build import build
    env = dict(os.environ, SBP_B200_LIBRARY=build(debug_bounds=True))
    r = subprocess.run([sys.executable, "-m", "pytest", *(os.path.join("tests", f) for f in FILES), "-x", "-q", "-m", "gpu", "-k", "not graph", "-p", "no:cacheprovider"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = r.stdout[-3000:] + r.stderr[-2000:]
    assert r.returncode == 0, tail
    last = r.stdout.strip().splitlines()[-1]
    assert " passed" in last and "failed" not in last, tail
    assert int(last.split(" passed")[0].split()[-1]) >= 600, last
