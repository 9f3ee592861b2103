"""Every kernel and tile of geocache_linear by itself (geocache_debug_set_linear), whatever the estimate would choose.

Small whole numbers, whose sums binary32 holds exactly in any order, bit for bit, with tokens, features and the summed axis one
off the tiles' edges.  And the accuracy of f32 results on products of one sign, where what the tensor cores cut off adds up:
their sums leave the accumulators after 16 instructions, of which each cuts at most 2^-22 of the sum so far, so a part is within
17 / 2 * 2^-22 of itself where it grows evenly, and within 16 * 2^-22 however it grows; P parts add (P + 1) / 2 * 2^-24, or P *
2^-24, the blocks of a cluster 8 * 2^-24, a scale two roundings.  One chain of all 512 instructions was 2.4e-5 (bf16) and 4.7e-5
(f16) off, eight and fifteen times the bound."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


@pytest.fixture
def gc(lib):
    yield lib
    lib.debug_set_linear()


def _whole(shape, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device=DEV).float()


def _rows(t, dtype):
    """rows of whole 16 bytes in a wider buffer of threes"""
    per = 16 // dtype.itemsize
    buf = torch.full((t.shape[0], (t.shape[1] + per - 1) // per * per + per), 3.0, device=DEV).to(dtype)
    buf[:, :t.shape[1]] = t.to(dtype)
    return buf[:, :t.shape[1]]


def _compare(gc, T, K, N, dtype, gated, od, taken=None):
    rows = N * (2 if gated else 1)
    x, w, bias, residual = _whole((T, K), T + K), _whole((rows, K), N + K), _whole((rows,), N), _whole((T, N), T)
    one = dict(x_scale=torch.ones(T, device=DEV), weight_scale=torch.ones(rows, device=DEV)) if dtype is E4M3 else {}
    z = x.double() @ w.double().T + bias.double()
    want = ((z[:, :N] * z[:, N:] if gated else z) + residual.double()).float().to(od)
    out = torch.full((T + 1, N + 3), 7.0, device=DEV, dtype=od)
    gc.linear(_rows(x, dtype), _rows(w, dtype), bias, None, gated, residual.to(od), out=out[:T, 1:1 + N], **one)
    if taken is not None:
        assert gc.debug_last_linear() == taken
    assert torch.equal(out[:T, 1:1 + N], want), (T, K, N, dtype, gated, od)
    assert (out[T] == 7).all() and (out[:, 0] == 7).all() and (out[:, 1 + N:] == 7).all()


TYPES = [(BF16, BF16), (BF16, F32), (F16, F16), (E4M3, BF16), (E4M3, F32)]


@pytest.mark.parametrize("splits", range(1, 9))
@pytest.mark.parametrize("tokens", [16, 32, 64])
def test_tiles(gc, tokens, splits):
    gc.debug_set_linear(gc.LINEAR_TILES, tokens, splits)
    for (dtype, od), gated in itertools.product(TYPES, (False, True)):
        chunk = 128 // dtype.itemsize
        # as many chunks as blocks, one more, and some times as many: stages of one and of two, a last block with fewer
        for K in (splits * chunk, splits * chunk + 1, splits * 7 * chunk - 3):
            for T, N in ((1, 1), (tokens - 1, 63), (tokens, 129), (tokens + 1, 65), (3 * tokens + 5, 200)):
                _compare(gc, T, K, N, dtype, gated, od, (gc.LINEAR_TILES, tokens, splits))


@pytest.mark.parametrize("features", [128, 256])
def test_pairs(gc, features):
    gc.debug_set_linear(gc.LINEAR_PAIRS, features)
    for (dtype, od), gated in itertools.product(TYPES, (False, True)):
        if features == 256 and od is F32:
            continue
        chunk = 128 // dtype.itemsize
        for K in (1, chunk, chunk + 1, 2 * chunk, 13 * chunk - 1):
            for T, N in ((1, 1), (127, 64), (129, 127), (255, 129), (257, 255), (600, 257), (1300, 520)):
                _compare(gc, T, K, N, dtype, gated, od, (gc.LINEAR_PAIRS, features, 0))


def test_few_features(gc):
    gc.debug_set_linear(gc.LINEAR_FEW_FEATURES)
    for dtype, od in TYPES:
        chunk = 128 // dtype.itemsize
        for K in (1, chunk, chunk + 1, 21 * chunk - 1):
            for T, N in ((1, 1), (127, 16), (129, 17), (257, 64), (20000, 33)):
                _compare(gc, T, K, N, dtype, False, od, (gc.LINEAR_FEW_FEATURES, 0, 0))


KERNELS = [(1, 16, 1), (1, 16, 8), (1, 32, 3), (1, 64, 1), (1, 64, 8), (2, 128, 1), (3, 0, 1)]


def _one_sign(gc, x, w, kernel, size, blocks, **one):
    T, N, K = 300, 40, x.shape[1]
    y = float((x.double() * w.double()).sum())
    if one:
        one = dict(x_scale=torch.full((T,), 0.75, device=DEV), weight_scale=torch.full((N,), 1.5, device=DEV))
        y *= 1.125
    gc.debug_set_linear(kernel, size, blocks)
    got = gc.linear(x.expand(T, K), w.expand(N, K), out_dtype=F32, **one).double()
    assert (got == got[0, 0]).all()
    return abs(got[0, 0].item() - y) / y


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("kernel,size,blocks", KERNELS)
def test_f32_results_of_one_sign(gc, kernel, size, blocks, dtype):
    K = 8192 * blocks   # 32 parts a block
    g = torch.Generator(device=DEV).manual_seed(K)
    x, w = ((torch.rand((1, K), generator=g, device=DEV) + 0.5).to(dtype) for _ in range(2))
    err = _one_sign(gc, x, w, kernel, size, blocks)
    assert err <= 17 / 2 * 2.0 ** -22 + 33 / 2 * 2.0 ** -24 + 8 * 2.0 ** -24 + 2 * 2.0 ** -24, err


@pytest.mark.parametrize("kernel,size,blocks", KERNELS)
def test_f32_results_of_8_bit_rows_of_one_sign(gc, kernel, size, blocks):
    # over a thousand sizes of products, so that the sums are not exact in 24 bits
    K = 16384 * blocks
    g = torch.Generator(device=DEV).manual_seed(K)
    x, w = (torch.exp2(10 * torch.rand((1, K), generator=g, device=DEV) - 5).to(E4M3) for _ in range(2))
    err = _one_sign(gc, x, w, kernel, size, blocks, scaled=True)
    assert err <= 16 * 2.0 ** -22 + 32 * 2.0 ** -24 + 8 * 2.0 ** -24 + 2 * 2.0 ** -24, err


def test_the_estimate_takes_every_kernel(gc):
    """Sizes that the estimate sends to each kind of tile, with the kernel that it takes on 152 SMs: a new estimate has to bring
    other sizes with it."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 152:
        pytest.skip("the choice depends on the number of SMs")
    for (T, K, N, dtype, gated, od), want in (
            ((1, 2048, 300, BF16, False, BF16), (1, 16, 8)), ((60, 6928, 1470, E4M3, False, BF16), (1, 32, 7)),
            ((374, 2600, 431, BF16, False, BF16), (1, 32, 4)), ((27, 112832, 19161, E4M3, False, BF16), (1, 32, 2)),
            ((81, 6096, 1831, BF16, False, BF16), (1, 32, 6)), ((265, 11744, 932, E4M3, True, F32), (1, 64, 4)),
            ((1298, 20880, 3, E4M3, False, BF16), (1, 64, 8)), ((12722, 416, 6, E4M3, True, F32), (1, 64, 1)),
            ((33, 43648, 6966, BF16, True, F32), (1, 64, 3)), ((4388, 16, 82, E4M3, True, BF16), (1, 32, 1)),
            ((300, 2048, 8192, BF16, False, BF16), (2, 256, 0)), ((9000, 512, 2048, E4M3, True, F32), (2, 128, 0)),
            ((9000, 2048, 2048, BF16, False, BF16), (2, 256, 0)), ((30000, 512, 40, F16, False, F32), (3, 0, 0))):
        _compare(gc, T, K, N, dtype, gated, od, want)
