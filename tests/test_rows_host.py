"""Refusals of geocache_add_rms_norm, geocache_quantize_rows and geocache_linear (no GPU needed: arguments are checked
before anything is launched)."""
import ctypes

import pytest

from paper_2608_13255_gb300 import build as gbuild

M = 1 << 20


@pytest.fixture(scope="module")
def gc():
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _ref(x):
    return None if x is None else ctypes.byref(x)


def test_add_rms_norm_checks_arguments(gc):
    L, T, C = gc.load(), 10, 64

    def rows(at, stride=C):
        return gc.Rows(at, stride)

    def call(x=rows(M), r=rows(2 * M), ro=rows(3 * M), out=rows(4 * M), T=T, C=C, dtype=1, rd=1, w=64 * M, eps=1e-6,
             scale=None):
        return L.geocache_add_rms_norm(_ref(x), _ref(r), _ref(ro), _ref(out), T, C, dtype, rd, w, eps, scale, None)

    assert call(T=-1) == gc.ESHAPE and call(T=2 ** 31) == gc.ESHAPE
    assert call(C=0) == gc.ESHAPE and call(C=65537) == gc.ESHAPE
    assert call(dtype=3) == gc.EDTYPE and call(dtype=-1) == gc.EDTYPE
    assert call(rd=2) == gc.EDTYPE and call(rd=3) == gc.EDTYPE and call(dtype=0, rd=1) == gc.EDTYPE
    for eps in (-1.0, float("nan"), float("inf"), 1e300):
        assert call(eps=eps) == gc.EINVAL
    assert call(r=None) == gc.EINVAL and call(ro=None) == gc.EINVAL
    assert call(x=None) == gc.EINVAL and call(out=None) == gc.EINVAL and call(x=rows(None)) == gc.EINVAL
    assert call(x=rows(M + 1)) == gc.EINVAL and call(w=64 * M + 2) == gc.EINVAL and call(scale=65 * M + 1) == gc.EINVAL
    assert call(x=rows(M, -1)) == gc.ESHAPE and call(x=rows(M, 2 ** 39)) == gc.ESHAPE
    # rows of an output that overlap each other
    assert call(out=rows(4 * M, 63)) == gc.EALIAS and call(ro=rows(3 * M, 0)) == gc.EALIAS
    # an output over a part of an input, of the other output, of the weight or of the scales
    assert call(out=rows(M + 16)) == gc.EALIAS and call(ro=rows(2 * M + 2)) == gc.EALIAS
    assert call(out=rows(M, 2 * C)) == gc.EALIAS
    assert call(out=rows(3 * M)) == gc.EALIAS and call(out=rows(2 * M), ro=rows(2 * M)) == gc.EALIAS
    assert call(w=4 * M + 64) == gc.EALIAS and call(w=3 * M) == gc.EALIAS
    for at in (M, 2 * M, 3 * M, 4 * M, 64 * M):
        assert call(scale=at) == gc.EALIAS
    # 8-bit rows over the 16-bit rows they come from; a residual in f32 over rows of 16 bits
    assert call(out=rows(M), scale=65 * M) == gc.EALIAS
    assert call(rd=0, ro=rows(M)) == gc.EALIAS and "overlaps" in gc.last_error()
    assert call(T=0, x=None, out=None) == gc.OK
    assert gc.last_launches() == 0


def test_quantize_rows_checks_arguments(gc):
    L, T, C = gc.load(), 10, 64

    def call(x=gc.Rows(M, C), out=gc.Rows(2 * M, C), T=T, C=C, dtype=1, scale=3 * M):
        return L.geocache_quantize_rows(_ref(x), _ref(out), T, C, dtype, scale, None)

    assert call(T=-1) == gc.ESHAPE and call(C=0) == gc.ESHAPE and call(C=65537) == gc.ESHAPE
    assert call(dtype=3) == gc.EDTYPE
    assert call(scale=None) == gc.EINVAL and call(x=None) == gc.EINVAL and call(out=None) == gc.EINVAL
    assert call(out=gc.Rows(M, C)) == gc.EALIAS and call(out=gc.Rows(M, 2 * C)) == gc.EALIAS
    assert call(scale=M) == gc.EALIAS and call(scale=2 * M) == gc.EALIAS
    assert call(out=gc.Rows(2 * M, 63)) == gc.EALIAS
    assert call(T=0, scale=None) == gc.OK
    assert gc.last_launches() == 0


def test_binding_of_rows_checks_tensors(gc):
    import torch
    x = torch.zeros((4, 64))
    for f in (gc.add_rms_norm, gc.quantize_rows):
        with pytest.raises(ValueError):
            f(x)
        with pytest.raises(TypeError):
            f(x.double())
        with pytest.raises(TypeError):
            f(x.to(torch.float8_e4m3fn))
        with pytest.raises(TypeError):
            f([[1.0]])


def test_linear_checks_arguments(gc):
    L, T, K, N = gc.load(), 10, 64, 32

    def rows(at, stride):
        return gc.Rows(at, stride)

    def call(x=rows(M, K), w=rows(2 * M, K), r=None, out=rows(4 * M, N), T=T, K=K, N=N, dtype=1, od=1, act=0, gated=0,
             bias=None, xs=None, ws=None):
        return L.geocache_linear(_ref(x), _ref(w), _ref(r), _ref(out), T, K, N, dtype, od, act, gated, bias, xs, ws, None)

    assert call(T=-1) == gc.ESHAPE and call(T=2 ** 31 - 1) == gc.ESHAPE
    for n in (0, 2 ** 20 + 1, -8):
        assert call(K=n) == gc.ESHAPE and call(N=n) == gc.ESHAPE
    assert call(dtype=0) == gc.EDTYPE and call(dtype=4) == gc.EDTYPE
    assert call(od=2) == gc.EDTYPE and call(dtype=2, od=1) == gc.EDTYPE and call(od=3) == gc.EDTYPE
    assert call(dtype=3, od=3, xs=8 * M, ws=9 * M) == gc.EDTYPE
    assert call(act=4) == gc.EINVAL and call(act=-1) == gc.EINVAL
    assert call(dtype=3) == gc.EINVAL and call(dtype=3, xs=8 * M) == gc.EINVAL and call(dtype=3, ws=9 * M) == gc.EINVAL
    assert call(xs=8 * M) == gc.EINVAL and call(ws=9 * M) == gc.EINVAL
    assert call(bias=8 * M + 2) == gc.EINVAL and call(dtype=3, xs=8 * M + 1, ws=9 * M) == gc.EINVAL
    assert call(x=None) == gc.EINVAL and call(w=None) == gc.EINVAL and call(out=None) == gc.EINVAL
    assert call(r=rows(None, N)) == gc.EINVAL and call(out=rows(4 * M + 1, N)) == gc.EINVAL
    # operands that the copies cannot take
    assert call(x=rows(M + 8, K)) == gc.EINVAL and call(w=rows(2 * M + 8, K)) == gc.EINVAL
    assert call(x=rows(M, 68)) == gc.EINVAL and call(dtype=3, x=rows(M, 72), xs=8 * M, ws=9 * M) == gc.EINVAL
    assert call(x=rows(M, -8)) == gc.ESHAPE and call(w=rows(2 * M, 2 ** 39)) == gc.ESHAPE
    assert call(out=rows(4 * M, 31)) == gc.EALIAS
    assert call(out=rows(M, N)) == gc.EALIAS and call(out=rows(2 * M, N)) == gc.EALIAS
    # beside the weights, but over the gates' rows
    at = 2 * M + 2 * N * K
    assert call(out=rows(at, N), gated=1) == gc.EALIAS
    assert call(r=rows(4 * M + 2, N)) == gc.EALIAS and call(r=rows(4 * M, 2 * N)) == gc.EALIAS
    assert call(bias=4 * M) == gc.EALIAS and call(dtype=3, xs=4 * M, ws=9 * M) == gc.EALIAS
    assert call(dtype=3, xs=8 * M, ws=4 * M) == gc.EALIAS
    assert call(T=0, x=None, w=None, out=None) == gc.OK
    assert gc.last_launches() == 0


def test_binding_of_linear_checks_tensors(gc):
    import torch
    x, w = torch.zeros((4, 64)), torch.zeros((32, 64))
    with pytest.raises(ValueError):
        gc.linear(x.bfloat16(), w.bfloat16(), out=x.bfloat16())
    with pytest.raises(TypeError):
        gc.linear(x.double(), w.double(), out=x)
    with pytest.raises(ValueError):
        gc.linear(x, w[:31], gated=True)
    with pytest.raises(TypeError):
        gc.linear(x, w, out=x, out_dtype=torch.float16)
