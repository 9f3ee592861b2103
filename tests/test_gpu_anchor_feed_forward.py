"""The example's block with a feed-forward (examples/anchor_attention.py --ff): its way back to the latents is the library's
product into f32, compared with 64 bits on the rows that it is given.  Tolerance: that of the products of
test_gpu_linear.py, S (steps 2^-22 + 16 * 2^-24) with S = sum |x w|; 16-bit rounding of x0 would be 2^-9 of it."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    spec = importlib.util.spec_from_file_location("anchor_attention", os.path.join(ROOT, "examples", "anchor_attention.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("views", [[0, 3], [0, 1, 2, 3, 4, 5]], ids=str)
def test_back_to_the_latents(ex, views, eight_bit, monkeypatch):
    w = ex.synth.make_workload("tiny", B=2)
    block = ex.Block(w, 4, 2, 64, ff=320, eight_bit=eight_bit)
    x = torch.randn((w.B, len(views), w.C, w.H, w.W), generator=torch.Generator(device="cuda").manual_seed(3),
                    device="cuda").to(torch.bfloat16)
    seen = []
    forward = block.feed_forward
    monkeypatch.setattr(block, "feed_forward", lambda rows: seen.append(forward(rows)) or seen[-1])
    got = block(x, views).permute(0, 1, 3, 4, 2).reshape(-1, w.C).double()
    ex.gc.device_status()
    place, rows = block.rows(tuple(views))[0], seen[0].double()
    want, size = rows @ block.back.double(), rows.abs() @ block.back.double().abs()
    steps = rows.shape[1] * 2 // 32
    assert ((got[place] - want).abs() <= size * (steps * 2.0 ** -22 + 16 * 2.0 ** -24)).all()
    rest = torch.ones(got.shape[0], dtype=torch.bool, device="cuda")
    rest[place] = False
    assert not got[rest].any()
