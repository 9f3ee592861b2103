"""The first calls of a process on rows made inside a stream capture: what a kernel's first launch sets up must not need
an uncaptured call before it."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys
sys.path.insert(0, %r)
import torch
from paper_2608_13255_gb300 import geocache as gc
x = torch.randn(300, 512, device="cuda").bfloat16()
y = torch.randn(6000, 512, device="cuda").bfloat16()
w = torch.randn(1024, 512, device="cuda").bfloat16()
b = torch.randn(1024, device="cuda")
torch.cuda.synchronize()
out = {}
def calls():
    out["norm"] = gc.add_rms_norm(x, x)[0]
    out["rows"], out["scale"] = gc.quantize_rows(x)
    out["few"] = gc.linear(x, w, bias=b, activation="gelu")
    out["many"] = gc.linear(y, w)
    out["f32"] = gc.linear(y, w, gated=True, activation="silu", out_dtype=torch.float32)
    out["split"] = gc.linear(x[:1], w)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
got = {k: v.clone() for k, v in out.items()}
calls()
gc.device_status()
for k, v in out.items():
    assert torch.equal(got[k].view(torch.uint8), v.view(torch.uint8)), k
print("same bits")
"""


def test_first_calls_captured():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    r = subprocess.run([sys.executable, "-c", CODE % ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same bits" in r.stdout, r.stderr[-2000:]
