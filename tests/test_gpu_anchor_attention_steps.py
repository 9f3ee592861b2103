"""The example's attention block (examples/anchor_attention.py) step by step:
the norms with the rotation and the attention each against 64 bits from the
values that they were given, with the tolerances of their own tests, and the
block's result as their composition bit for bit.

Tolerances.  Norm and rotation: 2^-19 (|a| + |b|) of a pair for the binary32
arithmetic and half a unit (2^-8) of bf16.  Attention: the weights' rounding and
their binary32 arithmetic, (2^-8 + 2^-12) sum_j p_j |v_j|, and the output's own
rounding."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = torch.finfo(torch.bfloat16).eps / 2


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


@pytest.mark.parametrize("heads,kv_heads,D", [(4, 2, 16), (4, 4, 64), (6, 2, 80)])
@pytest.mark.parametrize("views", [[0, 3], [1, 4], [0, 1, 2, 3, 4, 5]], ids=str)
def test_block_step_by_step(ex, views, heads, kv_heads, D):
    gc = ex.gc
    w = ex.synth.make_workload("tiny", B=2)
    block = ex.Block(w, heads, kv_heads, D)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((w.B, len(views), w.C, w.H, w.W), generator=g, device="cuda").to(torch.bfloat16)
    qkv, place, slots, plan = block.qkv(x, tuple(views))
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    before = qkv.clone()
    # the tokens keep their slots of the full layout: view, row, column
    token = place % (len(views) * w.H * w.W)
    assert torch.equal(slots.long(), torch.tensor(views, device="cuda")[token // (w.H * w.W)] * (w.H * w.W) + token % (w.H * w.W))
    gc.qk_norm_rope(q, k, block.table, slots, block.q_weight, block.k_weight, q_out=q, k_out=k)
    cs = torch.view_as_complex(block.table.double())[slots.long()][:, None]
    for got, raw, weight in ((q, before[:, :heads], block.q_weight), (k, before[:, heads:heads + kv_heads], block.k_weight)):
        y = raw.double()
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight.double()
        z = torch.complex(y[..., :D // 2], y[..., D // 2:]) * cs
        ref, size = torch.cat([z.real, z.imag], -1), (y[..., :D // 2].abs() + y[..., D // 2:].abs()).repeat(1, 1, 2)
        assert bool(((got.double() - ref).abs() <= (1 + U) * 2.0 ** -19 * size + U * ref.abs() + 2.0 ** -25).all())
    assert torch.equal(v, before[:, heads + kv_heads:])
    out = gc.attention(plan, q, k, v)
    asset = place // (len(views) * w.H * w.W)
    for b in range(w.B):
        m = asset == b
        K, V = (t[m].double().transpose(0, 1).repeat_interleave(heads // kv_heads, 0) for t in (k, v))
        P = torch.softmax(q[m].double().transpose(0, 1) @ K.transpose(1, 2) * D ** -0.5, -1)
        ref, size = (P @ V).transpose(0, 1), (P @ V.abs()).transpose(0, 1)
        tol = (U + 2.0 ** -12) * size + U * (1 + U) * ref.abs()
        assert bool(((out[m].double() - ref).abs() <= tol).all())
    x0 = torch.zeros((w.B * len(views) * w.H * w.W, w.C), device="cuda")
    x0[place] = (out.reshape(len(place), -1) @ block.back).float()
    assert torch.equal(block(x, views), x0.view(w.B, len(views), w.H, w.W, w.C).permute(0, 1, 4, 2, 3))
    gc.device_status()
