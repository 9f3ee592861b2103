"""Refusals of geocache_debug_set_linear and of the products that the kernel that is set cannot take (no GPU needed)."""
import ctypes

import pytest

from paper_2608_13255_gb300 import build as gbuild

M = 1 << 20


@pytest.fixture
def gc():
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    yield geocache
    geocache.debug_set_linear()


def test_which_kernels_can_be_set(gc):
    for kernel, size, splits in ((-1, 0, 0), (4, 0, 0), (1, 0, 1), (1, 128, 1), (1, 48, 2), (1, 16, 0), (1, 64, 9), (2, 64, 0), (2, 512, 0)):
        with pytest.raises(gc.GeocacheError) as e:
            gc.debug_set_linear(kernel, size, splits)
        assert e.value.status == gc.EINVAL
    for kernel, size, splits in ((1, 16, 1), (1, 32, 8), (2, 128, 0), (2, 256, 0), (3, 0, 0), (0, 0, 0)):
        gc.debug_set_linear(kernel, size, splits)
    assert gc.load().geocache_debug_last_linear(None, None, None) == gc.EINVAL


def test_products_that_the_kernel_cannot_take(gc):
    L = gc.load()

    def call(T=10, K=64, N=32, od=1, gated=0):
        x, w, out = gc.Rows(M, K), gc.Rows(2 * M, K), gc.Rows(4 * M, N)
        return L.geocache_linear(ctypes.byref(x), ctypes.byref(w), None, ctypes.byref(out), T, K, N, 1, od, 0, gated, None, None, None, None)

    gc.debug_set_linear(gc.LINEAR_TILES, 16, 2)   # a chunk is 64 elements
    assert call() == gc.EINVAL and "cannot take" in gc.last_error()
    gc.debug_set_linear(gc.LINEAR_PAIRS, 256)
    assert call(od=0) == gc.EINVAL
    gc.debug_set_linear(gc.LINEAR_FEW_FEATURES)
    assert call(N=65) == gc.EINVAL and call(gated=1) == gc.EINVAL
    assert gc.last_launches() == 0
