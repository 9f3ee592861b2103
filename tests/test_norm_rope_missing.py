"""geocache_qk_norm_rope called from C without one of its tensors, or with one
whose strides are out of range: refused whatever the others are (each call in a
process of its own, since it must not take the caller down)."""
import subprocess
import sys

import pytest

from paper_2608_13255_gb300 import build as gbuild

CALL = """
import ctypes, sys
sys.path.insert(0, %r)
from paper_2608_13255_gb300 import geocache as gc
L, M = gc.load(), 1 << 20
x = [gc.Heads((i + 1) * M, 256, 64) for i in range(4)]
bad = %r
at = [None if (i, "none") in bad else ctypes.byref(x[i]) for i in range(4)]
for i, what in bad:
    if what == "data":
        x[i].data = None
    if what == "stride":
        x[i].token_stride = 1 << 62
sys.exit(-L.geocache_qk_norm_rope(*at, 10, 4, 4, 64, 1, 1, 1e-6, None, None, None, 0, 0, 0, None, None))
"""


@pytest.mark.parametrize("what", ["none", "data", "stride"])
@pytest.mark.parametrize("which", range(4), ids=["q", "k", "q_out", "k_out"])
def test_a_missing_tensor_is_refused(which, what):
    gbuild.build()
    res = subprocess.run([sys.executable, "-c", CALL % (gbuild.ROOT, [(which, what)])], capture_output=True, text=True)
    assert res.returncode == (2 if what == "stride" else 1), (res.returncode, res.stderr)  # -ESHAPE, -EINVAL
