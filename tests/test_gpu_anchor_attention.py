"""The attention block's operators used together (examples/anchor_attention.py):
the block's x0 of the anchors and of all views against the same block in plain
64-bit torch, and a whole loop of full and cached steps.

Tolerance.  Queries and keys are rounded to bf16 after the norm and the rotation
(2^-8 of themselves each), and a score is at most 1.7 sqrt(D) (norm weights up to
1.3), so for D = 16 it is off by at most 6.8 * 2^-7 = 0.053, a weight and the sum
of the weights by 5.5% each, and an output by 0.11 A with A = sum_j p_j |v_j|,
beside the roundings of the weights and of the output (2^-8 each) and of the
projection behind it."""
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


def _plain(block, x, views):
    """(x0, its tolerance) of the block in 64 bits, from the same projections."""
    w, Hq, Hk, D = block.w, block.Hq, block.Hk, block.D
    qkv, place, slots, _ = block.qkv(x, tuple(views))
    qkv = qkv.double()
    cs = torch.view_as_complex(block.table.double())[slots.long()][:, None]

    def turn(y, weight):
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight.double()
        z = torch.complex(y[..., :D // 2], y[..., D // 2:]) * cs
        return torch.cat([z.real, z.imag], -1)

    q, k, v = turn(qkv[:, :Hq], block.q_weight), turn(qkv[:, Hq:Hq + Hk], block.k_weight), qkv[:, Hq + Hk:]
    asset = place // (len(views) * w.H * w.W)
    out, size = torch.empty_like(q), torch.empty_like(q)
    for b in range(w.B):
        m = asset == b
        K, V = (y[m].transpose(0, 1).repeat_interleave(Hq // Hk, 0) for y in (k, v))
        P = torch.softmax(q[m].transpose(0, 1) @ K.transpose(1, 2) * D ** -0.5, -1)
        out[m], size[m] = (P @ V).transpose(0, 1), (P @ V.abs()).transpose(0, 1)
    back = block.back.double()
    x0 = torch.zeros((w.B * len(views) * w.H * w.W, w.C), dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(x0)
    x0[place] = out.reshape(len(place), -1) @ back
    tol[place] = (size.reshape(len(place), -1) * (0.11 + 2.0 ** -7)) @ back.abs() + 2.0 ** -8 * x0[place].abs()
    shape = lambda y: y.view(w.B, len(views), w.H, w.W, w.C).permute(0, 1, 4, 2, 3)  # noqa: E731
    return shape(x0), shape(tol)


@pytest.mark.parametrize("views", [[0, 3], [1, 4], [0, 1, 2, 3, 4, 5]], ids=str)
def test_block_matches_64_bit_reference(ex, views):
    w = ex.synth.make_workload("tiny", B=1)
    block = ex.Block(w, 4, 2, 16)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((w.B, len(views), w.C, w.H, w.W), generator=g, device="cuda").to(torch.bfloat16)
    got = block(x, views).double()
    ref, tol = _plain(block, x, views)
    err = (got - ref).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    assert float(ref.abs().max()) > 0.1  # the block does something
    bg = ~(block.valid[:, views] != 0)[:, :, None].expand_as(got)
    assert not bool(got[bg].any())  # background tokens take no part
    ex.gc.device_status()


def test_loop_is_reproducible_and_finite(ex):
    w = ex.synth.make_workload("tiny", B=2)
    block = ex.Block(w, 4, 4, 64)
    a, a0 = ex.run(block, 7)
    b, b0 = ex.run(block, 7)
    ex.gc.device_status()
    assert torch.equal(a, b) and torch.equal(a0, b0)
    assert bool(torch.isfinite(a.float()).all()) and float(a0.abs().max()) > 0.1


def test_all_anchors_equal_the_full_step(ex):
    # the a = N gate: the anchor forward of every view is the full forward
    w = ex.synth.make_workload("tiny", B=1)
    block = ex.Block(w, 4, 4, 64)
    x = torch.randn((w.B, w.N, w.C, w.H, w.W), device="cuda").to(torch.bfloat16)
    full = block(x, range(w.N))
    packed = torch.empty_like(x)
    ex.gc.pack_anchors(x, packed, list(range(w.N)))
    assert torch.equal(block(packed, tuple(range(w.N))), full)
