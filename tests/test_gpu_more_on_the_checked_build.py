"""pods_logp_chunk's kernels for many rows, its finite masks, the optimiser's smallest states and full tables once more on the checked
build of the library: computed indices are compared with their extents, and a violation raises PODS_STATUS_INTERNAL, which those tests
reject."""
import os
import subprocess
import sys

import pytest

from paper_2504_13818_b200.csrc import build as cuda_build

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("tests", ["tests/test_gpu_logp_many_rows.py", "tests/test_gpu_logp_finite_masks.py", "tests/test_gpu_adamw_small_states.py",
                                   "tests/test_gpu_adamw_tables.py"])
def test_on_the_checked_build(tests):
    lib = cuda_build.CHECKED_LIB
    sources = cuda_build.SOURCES + cuda_build.HEADERS
    if not os.path.exists(lib) or any(os.path.getmtime(f) > os.path.getmtime(lib) for f in sources):
        cuda_build.build(checked=True)
    out = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", tests],
                         cwd=ROOT, env=dict(os.environ, PODS_B200_LIBRARY=lib), capture_output=True, text=True, timeout=1500)
    assert out.returncode == 0, out.stdout[-3000:] + out.stderr[-1000:]
    assert " passed" in out.stdout
