"""8-bit rows bit for bit: geocache_quantize_rows defines scale = max(max |x| r, 2^-126) with r = 1 / 448 rounded to binary32, and
out = e4m3(x / scale), each operation rounded to nearest in binary32.  torch's product, its division of two binary32 tensors and
its conversion to float8_e4m3fn are these operations, so scales and elements have to be equal, also at the ties of e4m3."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TINY = 2.0 ** -126


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _equal(gc, x):
    q, scale = gc.quantize_rows(x)
    y = x.float()
    want = (y.abs().amax(-1) * torch.full((), 1.0 / 448.0, device=DEV)).clamp(min=TINY)
    assert torch.equal(scale, want)
    assert torch.equal(q.view(torch.uint8), (y / want[:, None]).to(E4M3).view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C", [(1, 1), (700, 8), (300, 263), (4001, 512), (300, 513), (200, 2047), (129, 2048), (40, 8191),
                                 (7, 16384), (3, 65536), (2, 65535)])
def test_equals_the_definition(gc, T, C, dtype):
    g = torch.Generator(device=DEV).manual_seed(T + C)
    _equal(gc, torch.randn((T, C), generator=g, device=DEV).to(dtype))
    # rows that are multiples of their ties: the largest is 448 k, the others (2 m + 1) k / 2 steps
    k = torch.randint(1, 4, (T, 1), generator=g, device=DEV).float()
    m = torch.randint(-448 * 4, 448 * 4 + 1, (T, C), generator=g, device=DEV).float() / 4
    m[:, 0] = 448
    _equal(gc, (m * k).clamp(-60000, 60000).to(dtype))
    _equal(gc, (m * k * 2.0 ** -17).to(dtype))


def test_every_number_of_16_bits(gc):
    # each value of f16 and bf16 against 300 largest ones, over the range of a row
    for dtype in (torch.float16, torch.bfloat16):
        every = torch.arange(0, 0x8000, device=DEV, dtype=torch.int32).to(torch.int16).view(dtype)
        every = every[every.isfinite()]
        g = torch.Generator(device=DEV).manual_seed(1)
        tops = every[torch.randint(1, every.numel(), (300,), generator=g, device=DEV)]
        rows = torch.cat([torch.minimum(every[None, :], tops[:, None]), tops[:, None]], 1)
        _equal(gc, rows)
        _equal(gc, rows[:, 1:].contiguous())  # of whole words


@pytest.mark.parametrize("exponent", [-149, -140, -130, -126, -122, -118, -110, -90, -70, -62, -60, -58, -40, 0, 60, 100, 118])
@pytest.mark.parametrize("C", [1001, 1024])
def test_scales_of_every_size(gc, C, exponent):
    g = torch.Generator(device=DEV).manual_seed(C)
    x = torch.randn((50, C), generator=g, device=DEV).clamp(-7, 7)
    _equal(gc, torch.ldexp(x.double(), torch.tensor(exponent, device=DEV)).float())


def test_zeros_keep_their_sign(gc):
    x = torch.tensor([[0.0, -0.0, 1.0, -1e-30, 1e-30, -0.0, 448.0, -448.0]], device=DEV)
    for t in (x, x.bfloat16(), x[:, :6], torch.cat([x, x[:, :1].expand(1, 600)], 1)):
        _equal(gc, t)
    zero = torch.tensor([[0.0, -0.0, 0.0, -0.0]], device=DEV)
    _equal(gc, zero)
