"""The matrix product with its epilogue against its definition in 64 bits.

Two kinds of inputs.  Small whole numbers, whose products and sums binary32 holds exactly in any order: results are
compared bit for bit, so every element has to be there once.  And normal ones, with these tolerances: S = sum |x_k w_k|
bounds every partial sum; the sums of one instruction (32 bytes of a row) are added to the accumulator with a rounding
or truncation of at most 2^-22 S, the partial sums of at most 16 parts with 2^-24 S each.  Scales and bias add four
roundings; an activation's slope is at most 1.13, and its own error at most 2^-20 of |z| (exponential and quotient of a
few units, the error function likewise).  The result adds half a step of its type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _rows(t, dtype, K, wide=0):
    """[T, K] of dtype with rows of whole 16 bytes (`wide` elements more), as they are in a wider buffer"""
    per = 16 // dtype.itemsize
    stride = (K + per - 1) // per * per + wide
    buf = torch.full((t.shape[0], stride), 3.0, device=DEV).to(dtype)
    buf[:, :K] = t.to(dtype)
    return buf[:, :K]


def _whole(shape, seed, most=3):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).float()


def _randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def _exact_case(gc, T, K, N, dtype, wide=0):
    x, w = _whole((T, K), T + K), _whole((N, K), N)
    one = {}
    if dtype is E4M3:
        one = dict(x_scale=torch.ones(T, device=DEV), weight_scale=torch.ones(N, device=DEV))
    xr, wr = _rows(x, dtype, K, wide), _rows(w, dtype, K, wide)
    want = x.double() @ w.double().T
    for od in (F32, BF16 if dtype is not F16 else F16):
        assert torch.equal(gc.linear(xr, wr, out_dtype=od, **one), want.float().to(od)), (T, K, N, od)


# around the tiles' edges in tokens (16, 128, 256), features (64, 128, 256) and the summed axis (32, 64, 128)
SHAPES = [(1, 16, 4), (1, 8, 1), (2, 48, 7), (4, 2048, 300), (15, 64, 128), (16, 72, 130), (17, 128, 64), (64, 2064, 513), (100, 320, 257),
          (127, 4096, 96), (128, 136, 128), (129, 640, 129), (255, 16, 255), (256, 512, 1536), (257, 1040, 640), (512, 192, 64),
          (1000, 400, 1000), (1025, 1600, 777), (3000, 208, 260), (2049, 4096, 2049), (5391, 80, 520), (20000, 64, 64),
          (7, 10240, 5000), (300, 8192, 12288)]


@pytest.mark.parametrize("dtype", [BF16, F16, E4M3], ids=["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("T,K,N", SHAPES)
def test_whole_numbers(gc, T, K, N, dtype):
    _exact_case(gc, T, K, N, dtype)


@pytest.mark.parametrize("dtype", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,N", [(1, 1, 1), (3, 17, 9), (200, 333, 129), (700, 1001, 1300)])
def test_lengths_that_are_no_whole_words(gc, T, K, N, dtype):
    # what lies behind a row in its buffer (threes) is not summed
    _exact_case(gc, T, K, N, dtype)
    _exact_case(gc, T, K, N, dtype, wide=64)


def _act(z, kind):
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return z * torch.special.ndtr(z)
    if kind == "gelu_tanh":
        return z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def _reference(x, w, N, act, gated, bias, residual, xs, ws):
    """(result, bound of its error before the last rounding) in 64 bits"""
    xd, wd = x.double(), w.double()
    if xs is not None:
        xd, wd = xd * xs.double()[:, None], wd * ws.double()[:, None]
    z, S = xd @ wd.T, xd.abs() @ wd.abs().T
    steps = -(-x.shape[1] * x.dtype.itemsize // 32)
    dz = S * (steps * 2.0 ** -22 + 16 * 2.0 ** -24) + z.abs() * 2.0 ** -22
    if bias is not None:
        z = z + bias.double()
        dz = dz + z.abs() * 2.0 ** -24
    if gated:
        v, g = z[:, :N], z[:, N:]
        a = _act(g, act)
        da = 1.13 * dz[:, N:] + g.abs() * 2.0 ** -20
        y = v * a
        dy = v.abs() * da + (a.abs() + da) * dz[:, :N] + y.abs() * 2.0 ** -24
    elif act is None:
        y, dy = z, dz
    else:
        y, dy = _act(z, act), 1.13 * dz + z.abs() * 2.0 ** -20
    if residual is not None:
        y = y + residual.double()
        dy = dy + (y.abs() + dy) * 2.0 ** -24
    return y, dy


def _check(got, y, dy, dtype, what=""):
    assert got.dtype is dtype
    half = 0.0 if dtype is F32 else torch.finfo(dtype).eps / 2
    floor = 2.0 ** -25 if dtype is F16 else 2.0 ** -134  # half a step of the subnormal numbers
    err, most = (got.double() - y).abs(), dy * (1 + half) + y.abs() * half + floor
    assert (err <= most).all(), "%s: %g" % (what, (err - most).max())


EPILOGUES = [dict(), dict(bias=True), dict(act="gelu"), dict(act="gelu_tanh", bias=True), dict(act="silu"), dict(residual=True),
             dict(act="gelu", bias=True, residual=True), dict(gated=True, act="gelu", bias=True),
             dict(gated=True, act="gelu_tanh", residual=True), dict(gated=True, act="silu", bias=True, residual=True),
             dict(gated=True, bias=True)]


@pytest.mark.parametrize("dtype,od", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (E4M3, BF16), (E4M3, F16), (E4M3, F32)],
                         ids=["bf16", "bf16-f32", "f16", "f16-f32", "e4m3-bf16", "e4m3-f16", "e4m3-f32"])
@pytest.mark.parametrize("T,K,N", [(1, 512, 70), (5, 1600, 512), (130, 640, 200), (700, 768, 900), (2600, 512, 1200), (1300, 1024, 1300),
                                   (5000, 512, 4104)])
def test_epilogues(gc, T, K, N, dtype, od):
    for i, e in enumerate(EPILOGUES):
        gated = e.get("gated", False)
        rows = N * (2 if gated else 1)
        x, w = _randn((T, K), 10 * i), _randn((rows, K), 10 * i + 1) * 2 * K ** -0.5
        xs = ws = None
        if dtype is E4M3:
            x, xs = gc.quantize_rows(x)
            w, ws = gc.quantize_rows(w)
        else:
            x, w = x.to(dtype), w.to(dtype)
        bias = _randn((rows,), 10 * i + 2) if e.get("bias") else None
        residual = _randn((T, N), 10 * i + 3).to(od) if e.get("residual") else None
        x, w = _rows(x, dtype, K), _rows(w, dtype, K)
        got = gc.linear(x, w, bias, e.get("act"), gated, residual, xs, ws, out_dtype=od)
        y, dy = _reference(x, w, N, e.get("act"), gated, bias, residual, xs, ws)
        _check(got, y, dy, od, str(e))
        # the same bits in a second call, in place of the residual, and beside other columns
        assert torch.equal(gc.linear(x, w, bias, e.get("act"), gated, residual, xs, ws, out_dtype=od), got)
        if residual is not None:
            r = residual.clone()
            assert torch.equal(gc.linear(x, w, bias, e.get("act"), gated, r, xs, ws, out=r), got)
        for shift in (1, 2, 8):
            wide = torch.full((T + 1, N + 17), 5.0, device=DEV, dtype=od)
            r = None
            if residual is not None:
                r = torch.zeros((T, N + 9), device=DEV, dtype=od)[:, 3:3 + N]
                r.copy_(residual)
            out = gc.linear(x, w, bias, e.get("act"), gated, r, xs, ws, out=wide[:T, shift:shift + N])
            assert torch.equal(out, got)
            assert (wide[T] == 5).all() and (wide[:, :shift] == 5).all() and (wide[:, shift + N:] == 5).all()


@pytest.mark.parametrize("dtype,od", [(BF16, BF16), (BF16, F32), (F16, F32), (E4M3, F16), (E4M3, F32)],
                         ids=["bf16", "bf16-f32", "f16-f32", "e4m3-f16", "e4m3-f32"])
@pytest.mark.parametrize("T,K,N", [(7999, 320, 1), (9001, 64, 13), (5000, 1000, 16), (20479, 512, 17), (24577, 2048, 64), (24576, 1552, 39),
                                   (39001, 528, 61), (60001, 256, 64)])
def test_few_features(gc, T, K, N, dtype, od):
    # tokens in one, two, three and more rounds of blocks an SM; the last block with one token or all
    _exact_case(gc, T, K, N, dtype)
    for i, e in enumerate([dict(), dict(bias=True), dict(act="gelu_tanh", bias=True, residual=True), dict(act="silu", residual=True)]):
        x, w = _randn((T, K), 10 * i), _randn((N, K), 10 * i + 1) * 2 * K ** -0.5
        xs = ws = None
        if dtype is E4M3:
            x, xs = gc.quantize_rows(x)
            w, ws = gc.quantize_rows(w)
        bias = _randn((N,), 10 * i + 2) if e.get("bias") else None
        residual = _randn((T, N), 10 * i + 3).to(od) if e.get("residual") else None
        x, w = _rows(x, dtype, K, 32), _rows(w, dtype, K, 16)
        got = gc.linear(x, w, bias, e.get("act"), False, residual, xs, ws, out_dtype=od)
        y, dy = _reference(x, w, N, e.get("act"), False, bias, residual, xs, ws)
        _check(got, y, dy, od, str(e))
        if residual is not None:
            r = residual.clone()
            assert torch.equal(gc.linear(x, w, bias, e.get("act"), False, r, xs, ws, out=r), got)
        for shift in (1, 4):
            wide = torch.full((T + 1, N + 17), 5.0, device=DEV, dtype=od)
            assert torch.equal(gc.linear(x, w, bias, e.get("act"), False, residual, xs, ws, out=wide[:T, shift:shift + N]), got)
            assert (wide[T] == 5).all() and (wide[:, :shift] == 5).all() and (wide[:, shift + N:] == 5).all()


def test_few_features_not_finite(gc):
    T, K, N = 12001, 128, 33
    x, w = _whole((T, K), 1), _whole((N, K), 2)
    x[70, 3] = float("nan")
    x[300, 3] = float("inf")
    w[:, 3] = 1.0
    w[9, 5] = float("nan")
    ref = gc.linear(torch.nan_to_num(x, 0.0, 0.0).to(BF16), torch.nan_to_num(w, 0.0).to(BF16), out_dtype=F32)
    got = gc.linear(x.to(BF16), w.to(BF16), out_dtype=F32)
    nan = torch.zeros((T, N), dtype=torch.bool, device=DEV)
    nan[70] = True
    nan[:, 9] = True
    inf = torch.zeros_like(nan)
    inf[300] = True
    inf &= ~nan
    assert got[nan].isnan().all() and (got[inf] == float("inf")).all() and torch.equal(got[~nan & ~inf], ref[~nan & ~inf])


@pytest.mark.parametrize("dtype", [BF16, E4M3], ids=["bf16", "e4m3"])
def test_extremes(gc, dtype):
    # the activations far from zero, and rows and columns that are not finite
    T, K, N = 150, 64, 140
    x, w = torch.zeros((T, K), device=DEV), torch.zeros((N, K), device=DEV)
    x[:, 0] = torch.linspace(-1, 1, T, device=DEV)
    w[:, 0] = 2.0 ** torch.linspace(-8, 8, N, device=DEV).round()
    one = {}
    if dtype is E4M3:
        one = dict(x_scale=torch.full((T,), 100.0, device=DEV), weight_scale=torch.full((N,), 10.0, device=DEV))
    x, w = x.to(dtype), w.to(dtype)
    for act in (None, "gelu", "gelu_tanh", "silu"):
        got = gc.linear(x, w, activation=act, out_dtype=F32, **one)
        y, dy = _reference(x, w, N, act, False, None, None, one.get("x_scale"), one.get("weight_scale"))
        _check(got, y, dy, F32, str(act))
    ref = gc.linear(x, w, out_dtype=F32, **one)
    x, w = x.float(), w.float()
    x[7, 3] = float("nan")
    w[9, 5] = float("nan")
    if dtype is not E4M3:
        x[8, 3] = float("inf")
    got = gc.linear(x.to(dtype), w.to(dtype), out_dtype=F32, **one)
    bad = torch.zeros((T, N), dtype=torch.bool, device=DEV)
    bad[7] = True
    bad[:, 9] = True
    if dtype is not E4M3:
        bad[8] = True  # (infinity times zero)
    assert got[bad].isnan().all() and torch.equal(got[~bad], ref[~bad])


def test_rows_behind_and_empty(gc):
    x, w = _whole((300, 64), 1).to(BF16), _whole((96, 64), 2).to(BF16)
    out = torch.full((310, 96), 9.0, device=DEV, dtype=BF16)
    gc.linear(x, w, out=out[:300])
    assert (out[300:] == 9).all()
    assert gc.linear(x[:0], w).shape == (0, 96) and gc.last_launches() == 0
    assert torch.equal(gc.linear(x[5:6].expand(40, 64), w), out[5:6].expand(40, 96))   # a row read many times
    assert torch.equal(gc.linear(x, w[3:4].expand(40, 64)), out[:300, 3:4].expand(300, 40))


def test_offsets_past_32_bits(gc):
    T, K, N = 3, 64, 64
    stride = 2 ** 31 + 64
    wide = torch.empty(2 * stride + K, device=DEV, dtype=BF16)
    x = torch.as_strided(wide, (T, K), (stride, 1))
    src, w = _whole((T, K), 1).to(BF16), _whole((N, K), 2).to(BF16)
    x.copy_(src)
    want = gc.linear(src, w)
    assert torch.equal(gc.linear(x, w), want)
    out = torch.as_strided(wide, (T, N), (stride, 1))
    gc.linear(src, w, out=out)
    assert torch.equal(out, want)


def test_streams_and_graph(gc):
    T, K, N = 300, 512, 512
    x, w1, w2 = _randn((T, K), 1).to(BF16), (_randn((N, K), 2) / 30).to(BF16), (_randn((K, N), 3) / 30).to(BF16)

    def chain(x, hidden, out, stream=None):
        gc.linear(x, w1, activation="silu", out=hidden, stream=stream)
        return gc.linear(hidden, w2, residual=x, out=out, stream=stream)

    def buffers():
        return torch.empty((T, N), device=DEV, dtype=BF16), torch.empty((T, K), device=DEV, dtype=BF16)

    want = chain(x, *buffers()).clone()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(4):  # two at once
        for st in streams:
            got.append(chain(x, *buffers(), stream=st))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    bufs, held = buffers(), x.clone()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            chain(held, *bufs)
            held.copy_(bufs[1])
    ref = x
    for i in range(4):
        graphs[i % 2].replay()
        ref = chain(ref, *buffers())
        assert torch.equal(held, ref)
    gc.device_status()


@pytest.mark.parametrize("T,K,N", [(4, 4096, 512), (512, 512, 1536), (300, 1024, 256), (2600, 2048, 1200), (6000, 512, 512),
                                   (30000, 2048, 40)])
def test_waits_that_run_out(gc, T, K, N):
    x, w = _randn((T, K), 1).to(BF16), _randn((N, K), 2).to(BF16)
    want = gc.linear(x, w)
    gc.device_status()
    for limit, drop in ((200_000, True), (1, False), (1, True)):
        late = False
        try:
            gc.debug_set_wait(limit, drop_first_copy=drop)
            first = gc.linear(x, w)
            gc.debug_set_wait(0, drop_first_copy=False)
            second = gc.linear(x, w)  # queued behind, before anything is waited for
            torch.cuda.synchronize()
            try:
                gc.device_status()
            except gc.GeocacheError as e:
                assert e.status == gc.ETIMEOUT
                late = True
        finally:
            gc.debug_set_wait(0, drop_first_copy=False)
        assert torch.equal(second, want)
        assert late if drop else (late or torch.equal(first, want))
    gc.device_status()
