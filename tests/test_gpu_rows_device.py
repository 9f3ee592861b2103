"""Rows on another device than the current one are refused before anything is launched (a machine with one GPU has no such
tensor: skipped there)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_rows_of_another_device():
    if torch.cuda.device_count() < 2:
        pytest.skip("needs a second device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache as gc
    here, there = torch.zeros((4, 64), device="cuda:0").bfloat16(), torch.zeros((4, 64), device="cuda:1").bfloat16()
    with torch.cuda.device(0):
        for call in (lambda: gc.add_rms_norm(there), lambda: gc.add_rms_norm(here, residual=there), lambda: gc.quantize_rows(there),
                     lambda: gc.linear(here, there), lambda: gc.linear(there, here),
                     lambda: gc.linear(here, here, bias=torch.zeros(4, device="cuda:1"))):
            with pytest.raises(ValueError, match="current device"):
                call()
