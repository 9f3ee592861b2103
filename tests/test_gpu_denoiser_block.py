"""A denoiser's block of the library's calls, as a program runs them: norm, projection to queries, keys and values, their
norms and rotation, attention, projection back into the residual, norm, feed-forward.  Each call is compared with its
definition in 64 bits on the inputs it was given (the tolerances are those of the single operators' tests; the attention's
and the rotation's stand in theirs), and the whole, captured and on several streams, with itself."""
import importlib.util
import os

import pytest
import torch

from test_gpu_linear import _check as check_linear
from test_gpu_linear import _reference as linear_reference
from test_gpu_norm_rows import F32 as NORM_REL
from test_gpu_norm_rows import _check as check_norm
from test_gpu_norm_rows import _check_quantised, _norm

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV, BF16 = "cuda", torch.bfloat16


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


class _Model:
    """Weights of a block, and its buffers and plan, kept as a program keeps them."""

    def __init__(self, gc, lens, H, D, F, eight):
        self.gc, self.H, self.D, self.F, self.eight, self.T = gc, H, D, F, eight, sum(lens)
        M = H * D
        g = torch.Generator(device=DEV).manual_seed(M + F)
        r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.norms = [1 + 0.1 * r(M) for _ in range(2)]
        self.w = {"qkv": r(3 * M, M) / M ** 0.5, "out": r(M, M) / M ** 0.5, "up": r(2 * F, M) / M ** 0.5,
                  "down": r(M, F) / F ** 0.5}
        self.scales = dict.fromkeys(self.w)
        for name, w in self.w.items():
            self.w[name] = w.to(BF16)
            if eight:
                self.w[name], self.scales[name] = gc.quantize_rows(self.w[name])
        self.bias = 0.1 * r(3 * M)
        self.table = gc.rope_table(self.T, D)
        self.plan = gc.attention_plan(lens, lens, H, H, D)
        self.seen = None

    def product(self, name, rows, scale, stream, **kw):
        if self.eight and scale is None:
            rows, scale = self.gc.quantize_rows(rows, stream=stream)
        out = self.gc.linear(rows, self.w[name], x_scale=scale, weight_scale=self.scales[name], stream=stream, **kw)
        if self.seen is not None:
            self.seen.append(("linear", name, rows, scale, kw, out))
        return out

    def norm(self, i, x, residual, stream):
        out, scale, kept = self.gc.add_rms_norm(x, residual, self.norms[i], quantize=self.eight, stream=stream)
        if self.seen is not None:
            self.seen.append(("norm", i, x, residual, out, scale, kept))
        return out, scale, x if kept is None else kept

    def __call__(self, x, added, stream=None, workspace=None):
        """The stream of rows x with `added` from the block before, through one block."""
        gc, H, D, M = self.gc, self.H, self.D, self.H * self.D
        rows, scale, kept = self.norm(0, added, x, stream)
        qkv = self.product("qkv", rows, scale, stream, bias=self.bias).view(self.T, 3 * H, D)
        q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
        q, k = gc.qk_norm_rope(q, k, self.table, q_out=q, k_out=k, stream=stream)
        heads = gc.attention(self.plan, q, k, v, stream=stream, workspace=workspace).reshape(self.T, M)
        kept = self.product("out", heads, None, stream, residual=kept)
        rows, scale, _ = self.norm(1, kept, None, stream)
        hidden = self.product("up", rows, scale, stream, activation="gelu_tanh", gated=True)
        return self.product("down", hidden, None, stream, residual=kept, out=kept)


def _rows(T, M, seed):
    return torch.randn((T, M), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(BF16)


CASES = [([1], 2, 64, 80, False), ([37, 0, 100], 4, 64, 304, True), ([700, 333], 8, 64, 1000, False), ([2048, 500], 4, 128, 768, True)]


@pytest.mark.parametrize("lens,H,D,F,eight", CASES, ids=lambda c: str(c).replace(" ", ""))
def test_each_call_of_a_block(ex, lens, H, D, F, eight):
    m = _Model(ex.gc, lens, H, D, F, eight)
    x, added = _rows(m.T, H * D, 1), _rows(m.T, H * D, 2)
    m.seen = []
    before = x.clone(), added.clone()
    m(x, added)
    ex.gc.device_status()
    assert torch.equal(x, before[0]) and torch.equal(added, before[1])  # (new outputs, but for the last)
    for call in m.seen:
        if call[0] == "norm":
            _, i, rows, residual, out, scale, kept = call
            h = rows
            if residual is not None:
                h = (rows.float() + residual.float()).to(BF16)
            if i == 0:  # (the second norm's rows have become the block's output)
                if residual is not None:
                    assert torch.equal(kept, h)
                y = _norm(h, m.norms[i], 1e-6)
                if eight:
                    _check_quantised(out, scale, y, NORM_REL)
                else:
                    check_norm(out, y, BF16)
        elif call[1] == "up":  # (the others' outputs are rotated or added to in place: below)
            _, name, rows, scale, kw, out = call
            y, dy = linear_reference(rows, m.w[name], F, kw["activation"], True, None, None, scale, m.scales[name])
            check_linear(out, y, dy, BF16, name)


@pytest.mark.parametrize("lens,H,D,F,eight", CASES, ids=lambda c: str(c).replace(" ", ""))
def test_products_that_later_calls_overwrite(ex, lens, H, D, F, eight):
    # the projections whose outputs are rotated or added to in place, looked at before that
    m = _Model(ex.gc, lens, H, D, F, eight)
    M = H * D
    rows, kept = _rows(m.T, M, 3), _rows(m.T, M, 4)
    hidden = _rows(m.T, F, 5)
    for name, x, kw in (("qkv", rows, dict(bias=m.bias)), ("out", rows, dict(residual=kept)), ("down", hidden, dict(residual=kept))):
        scale = None
        if eight:
            x, scale = ex.gc.quantize_rows(x)
        w = m.w[name]
        out = ex.gc.linear(x, w, x_scale=scale, weight_scale=m.scales[name], **kw)
        y, dy = linear_reference(x, w, out.shape[1], None, False, kw.get("bias"), kw.get("residual"), scale, m.scales[name])
        check_linear(out, y, dy, BF16, name)
        if "residual" in kw:
            r = kept.clone()
            kw["residual"] = r
            assert torch.equal(ex.gc.linear(x, w, x_scale=scale, weight_scale=m.scales[name], out=r, **kw), out)


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
def test_block_captured_and_on_streams(ex, eight):
    lens, H, D, F = [700, 333, 5], 8, 64, 1024
    m = _Model(ex.gc, lens, H, D, F, eight)
    x, added = _rows(m.T, H * D, 1), _rows(m.T, H * D, 2)
    want = m(x, added).clone()
    twice = m(want, added).clone()
    # on two streams at once, each with its workspace
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    spaces = [None if m.plan.workspace is None else torch.empty_like(m.plan.workspace) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, ws in zip(streams, spaces):
            got.append(m(x, added, stream=st, workspace=ws))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    # captured: two layers in a graph, replayed between eager calls
    held = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m(m(held, added), added)
    for _ in range(3):
        graph.replay()
        assert torch.equal(out, twice)
        assert torch.equal(m(x, added), want)
    held.copy_(want)
    graph.replay()
    assert torch.equal(out, m(m(want, added), added))
    ex.gc.device_status()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
def test_example_with_a_feed_forward(ex, eight):
    w = ex.synth.make_workload("tiny", B=2)
    block = ex.Block(w, 4, 2, 64, ff=320, eight_bit=eight)
    plain = ex.Block(w, 4, 2, 64)
    a, a0 = ex.run(block, 5)
    b, b0 = ex.run(block, 5)
    ex.gc.device_status()
    assert torch.equal(a, b) and torch.equal(a0, b0) and bool(torch.isfinite(a.float()).all())
    assert not torch.equal(ex.run(plain, 5)[1], a0)  # the feed-forward does something
