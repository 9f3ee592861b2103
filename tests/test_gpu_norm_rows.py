"""The norm with the residual's addition, and 8-bit rows, against their definition in 64 bits.

Tolerances.  A row's sum of squares is taken by chains of at most 64 elements a thread, 5 additions over a warp and 31
over warps: positive terms, so at most 100 roundings of 2^-24 relative, halved by the root; the root itself, the division
by C, the addition of eps, three products and the scale's division add at most 12 more.  A result of n bits adds half a
step."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
F32 = (50 + 12) * 2.0 ** -24   # of a normalised value before its last rounding, relative


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _randn(shape, seed, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _norm(h, weight, eps):
    h = h.double()
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return y if weight is None else y * weight.double()


def _check_quantised(q, scale, y, rel, what=""):
    want = (y.abs().amax(-1) / 448).clamp(min=2.0 ** -126)
    assert q.dtype is E4M3 and scale.dtype is torch.float32
    assert ((scale.double() - want).abs() <= (rel + 2.0 ** -23) * want).all(), what
    t = y / scale.double()[:, None]
    # half a step of e4m3: 2^-4 of the value, 2^-10 below its least normal number
    err, most = (q.double() - t).abs(), torch.clamp(t.abs() * 2.0 ** -4, min=2.0 ** -10) + t.abs() * 2 * (rel + 2.0 ** -22)
    assert (err <= most).all(), "%s: %g" % (what, (err - most).max())


def _check(got, y, dtype, what=""):
    assert got.dtype is dtype
    half = 0.0 if dtype is torch.float32 else torch.finfo(dtype).eps / 2
    floor = 2.0 ** -25 if dtype is torch.float16 else 0.0  # half a step of its subnormal numbers
    err, most = (got.double() - y).abs(), y.abs() * (half + F32 * (1 + half)) + floor
    assert (err <= most).all(), "%s: %g" % (what, (err - most).max())


SIZES = [(1, 1), (3, 7), (1, 8), (257, 9), (5, 64), (1000, 80), (33, 513), (300, 1600), (129, 2048), (7, 8192), (3, 8200),
         (2, 16384), (2, 40000), (1, 65536)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C", SIZES)
def test_norm(gc, T, C, dtype):
    x, res, w = _randn((T, C), 1, dtype), _randn((T, C), 2, dtype), 1 + 0.1 * _randn((C,), 3, torch.float32)
    res32 = res.float() * 1.001
    for residual in (None, res, res32):
        h, want = x, None
        if residual is not None:
            want = (x.float() + residual.float()).to(residual.dtype)
            h = want
        for weight in (None, w):
            for quantize in (False, True):
                out, scale, ro = gc.add_rms_norm(x, residual, weight, 1e-5, quantize=quantize)
                y = _norm(h, weight, 1e-5)
                if want is not None:
                    assert ro.dtype is want.dtype and torch.equal(ro, want)
                else:
                    assert ro is None
                if quantize:
                    _check_quantised(out, scale, y, F32)
                else:
                    assert scale is None
                    _check(out, y, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C", SIZES)
def test_quantize(gc, T, C, dtype):
    x = _randn((T, C), 4, dtype)
    q, scale = gc.quantize_rows(x)
    _check_quantised(q, scale, x.double(), 0.0)


@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("C", [96, 97])
def test_strides_and_alignment(gc, C, shift):
    # rows inside wider buffers, whose other elements stay as they are
    T, W = 37, 160
    dt = torch.bfloat16
    x, res = (_randn((T, W), s, dt)[:, shift:shift + C] for s in (1, 2))
    buf, buf8 = torch.full((T, W), 7.0, device=DEV, dtype=dt), torch.full((T, W), 3.0, device=DEV).to(E4M3)
    rbuf = torch.full((T, W), 5.0, device=DEV, dtype=dt)
    want = (x.float() + res.float()).to(dt)
    y = _norm(want, None, 1e-6)
    gc.add_rms_norm(x, res, out=buf[:, shift:shift + C], residual_out=rbuf[:, shift:shift + C])
    _check(buf[:, shift:shift + C], y, dt)
    assert torch.equal(rbuf[:, shift:shift + C], want)
    _, scale, _ = gc.add_rms_norm(x, res, out=buf8[:, shift:shift + C], residual_out=rbuf[:, shift:shift + C])
    _check_quantised(buf8[:, shift:shift + C], scale, y, F32)
    for b, v in ((buf, 7.0), (rbuf, 5.0), (buf8.float(), 3.0)):
        assert (b[:, :shift] == v).all() and (b[:, shift + C:] == v).all()
    q, s = gc.quantize_rows(x)
    _check_quantised(q, s, x.double(), 0.0)
    # a row read many times (stride 0), and a single row whose stride says nothing
    same = x[:1].expand(T, C)
    out, _, _ = gc.add_rms_norm(same)
    assert torch.equal(out, out[:1].expand(T, C))
    one = torch.as_strided(x, (1, C), (0, 1))
    assert torch.equal(gc.add_rms_norm(one)[0], out[:1])


def test_rows_behind_the_last_stay(gc):
    T, C = 5, 512
    x, out = _randn((T, C), 1, torch.float16), torch.full((T + 3, C), 9.0, device=DEV, dtype=torch.float16)
    gc.add_rms_norm(x, out=out[:T])
    assert (out[T:] == 9).all() and not (out[:T] == 9).all()
    scale = torch.full((T + 3,), 9.0, device=DEV)
    q, _ = gc.quantize_rows(x, scale=scale[:T])
    assert (scale[T:] == 9).all()
    assert gc.add_rms_norm(x[:0])[0].shape == (0, C)
    assert gc.last_launches() == 0


def test_in_place(gc):
    T, C = 65, 800
    x, res, w = _randn((T, C), 1, torch.bfloat16), _randn((T, C), 2, torch.bfloat16), _randn((C,), 3, torch.float32)
    out, _, ro = gc.add_rms_norm(x, res, w)
    a, b = x.clone(), res.clone()
    assert gc.add_rms_norm(a, b, w, out=a, residual_out=b)[0] is a
    assert torch.equal(a, out) and torch.equal(b, ro)
    a, b = x.clone(), res.clone()
    gc.add_rms_norm(a, b, w, out=b, residual_out=a)  # and the other way round
    assert torch.equal(b, out) and torch.equal(a, ro)
    with pytest.raises(gc.GeocacheError) as e:
        gc.add_rms_norm(x, res, out=x[:, :], residual_out=x[:, :])
    assert e.value.status == gc.EALIAS


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_rows_without_size_and_not_finite(gc, dtype):
    T, C = 9, 200
    x = _randn((T, C), 1, dtype)
    x[1] = 0
    x[2] = 0
    x[2, 7] = 1e-37
    x[3, 5] = float("nan")
    x[4, 9] = float("inf")
    x[5] = 1e-30
    out, _, _ = gc.add_rms_norm(x)
    q, s, _ = gc.add_rms_norm(x, quantize=True)
    assert (out[1] == 0).all() and (q[1].float() == 0).all() and s[1] == 2.0 ** -126
    assert out[3].isnan().all() and s[3].isnan() and q[3].float().isnan().all()
    # an infinity makes the root infinite: zeros beside it, and no number in its own place
    assert out[4, 9].isnan() and (out[4, :9] == 0).all() and q[4].float().isnan()[9]
    ok = [0, 5, 6, 7, 8]
    y = _norm(x, None, 1e-6)
    _check(out[ok], y[ok], dtype)
    _check_quantised(q[ok], s[ok], y[ok], F32)
    q, s = gc.quantize_rows(x)
    assert (q[1].float() == 0).all() and s[1] == 2.0 ** -126
    _check_quantised(q[[0, 2, 5, 6]], s[[0, 2, 5, 6]], x[[0, 2, 5, 6]].double(), 0.0)
    assert s[3].isnan() and s[4].isinf() and (q[4, :9].float() == 0).all() and q[4, 9].float().isnan()
    # without eps a row of zeros has no norm
    assert gc.add_rms_norm(x[1:2], eps=0.0)[0].isnan().all()


def test_streams_and_graph(gc):
    T, C = 300, 640
    x, res, w = _randn((T, C), 1, torch.bfloat16), _randn((T, C), 2, torch.bfloat16), _randn((C,), 3, torch.float32)
    want = gc.add_rms_norm(x, res, w, quantize=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = gc.add_rms_norm(x, res, w, quantize=True, stream=st)
    st.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    bufs = [torch.empty_like(t) for t in want]
    stream = res.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gc.add_rms_norm(x, stream, w, out=bufs[0], scale=bufs[1], residual_out=stream)
        gc.quantize_rows(stream, out=bufs[2].view(E4M3)[:, :C], scale=bufs[1])
    r = res
    for _ in range(3):
        graph.replay()
        r = (x.float() + r.float()).to(torch.bfloat16)
        assert torch.equal(stream, r)
        q, s = gc.quantize_rows(r)
        assert torch.equal(bufs[1], s) and torch.equal(bufs[2].view(torch.uint8)[:, :C], q.view(torch.uint8))


def test_offsets_past_32_bits(gc):
    # 2^32 elements between the rows' ends
    C, T = 64, 3
    stride = 2 ** 31 + 64
    wide = torch.empty(2 * stride + C, device=DEV, dtype=torch.bfloat16)
    x = torch.as_strided(wide, (T, C), (stride, 1))
    src = _randn((T, C), 1, torch.bfloat16)
    x.copy_(src)
    assert torch.equal(gc.add_rms_norm(x)[0], gc.add_rms_norm(src)[0])
    want = gc.add_rms_norm(src)[0]
    gc.add_rms_norm(x, out=x)
    assert torch.equal(x, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C", [(2999, 520), (3001, 520), (3100, 1811), (4000, 8184)])
def test_many_rows(gc, T, C, dtype):
    # the division of a row over threads depends on the number of rows
    x, res, w = _randn((T, C), 1, dtype), _randn((T, C), 2, dtype), 1 + 0.1 * _randn((C,), 3, torch.float32)
    for residual in (None, res):
        h = x if residual is None else (x.float() + res.float()).to(dtype)
        y = _norm(h, w, 1e-5)
        out, _, ro = gc.add_rms_norm(x, residual, w, 1e-5)
        _check(out, y, dtype)
        assert residual is None or torch.equal(ro, h)
        q, scale, _ = gc.add_rms_norm(x, residual, w, 1e-5, quantize=True)
        _check_quantised(q, scale, y, F32)
        # few of the rows by themselves: the other division, sums in another order
        some = gc.add_rms_norm(x[:50], None if residual is None else residual[:50], w, 1e-5)[0]
        _check(some, y[:50], dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C", [(40, 513), (700, 1031), (5, 8191), (9, 8193), (3, 16383), (3, 16385), (2, 65535)])
def test_rows_that_are_no_whole_words(gc, T, C, dtype):
    # single elements, from and into rows at every alignment, with a residual in place
    x = _randn((T, C + 3), 1, dtype)[:, 1:1 + C]
    res, w = _randn((T, C), 2, dtype), 1 + 0.1 * _randn((C,), 3, torch.float32)
    for residual in (None, res, res.float() * 1.001):
        h = x if residual is None else (x.float() + residual.float()).to(residual.dtype)
        y = _norm(h, w, 1e-5)
        kept = None if residual is None else residual.clone()
        out = torch.full((T, C + 5), 7.0, device=DEV, dtype=dtype)
        gc.add_rms_norm(x, kept, w, 1e-5, out=out[:, 2:2 + C], residual_out=kept)
        _check(out[:, 2:2 + C], y, dtype)
        assert (out[:, :2] == 7).all() and (out[:, 2 + C:] == 7).all()
        assert residual is None or torch.equal(kept, h)
        q, scale, _ = gc.add_rms_norm(x, residual, w, 1e-5, quantize=True)
        _check_quantised(q, scale, y, F32)
    q, scale = gc.quantize_rows(x)
    _check_quantised(q, scale, x.double(), 0.0)
