"""The erf GELU of geocache_linear's epilogue on f32 and f16 results, against 64 bits.

One nonzero product a sum, with a factor of one: the sums are the inputs, exactly.  The result is max(z, 0) - |z| Q(|z|),
Q(m) = erfc(m / sqrt 2) / 2 = e^(-m^2 / 2) t P(t) with t = 1 / (1 + 0.36 m).  Relative to Q: the polynomial as it is rounded is
within 1.1e-7; its evaluation in binary32 adds sum_k (2 k + 1) |c_k| t^k 2^-24 <= 1.01e-6; t (two roundings and an approximate
inverse within 2^-23, times d ln Q / d ln t <= 2.22) adds 5.3e-7; the exponential 2^-22, its argument's three roundings
m^2 / 2 * 3 * 2^-24 <= 9e-8 m^2, four products 2^-22.  Together 2.2e-6 + 9e-8 m^2 of |z| Q; the subtraction rounds the result
once."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


# tiles of one block and of a cluster, few features, pairs of SMs
@pytest.mark.parametrize("T,K,N", [(600, 16, 100), (40, 4096, 128), (45000, 64, 8), (20000, 512, 1024)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("gated", [False, True], ids=["", "gated"])
def test_gelu_of_f32_results(gc, T, K, N, dtype, gated):
    every = torch.arange(0, 0x8000, device=DEV, dtype=torch.int32).to(torch.int16).view(dtype)
    every = every[(every <= 12) & (every > 2.0 ** -20)]
    every = torch.cat([every, -every]).sort().values
    z = every[torch.arange(T * 16, device=DEV) * every.numel() // (T * 16)].view(T, 16)   # [T, 16], evenly from all of them
    x = torch.zeros((T, K), device=DEV, dtype=dtype)
    x[:, K - 16:] = z
    pick = torch.arange(N, device=DEV) % 16
    w = torch.zeros((N, K), device=DEV, dtype=dtype)
    w[torch.arange(N, device=DEV), K - 16 + pick] = 1
    bias = None
    if gated:   # the values are ones
        w, bias = torch.cat([torch.zeros_like(w), w]), torch.cat([torch.ones(N, device=DEV), torch.zeros(N, device=DEV)])
    got = gc.linear(x, w, bias, "gelu", gated, out_dtype=torch.float32).double()
    zd = z.double()[:, pick]
    m = zd.abs()
    tail = m * 0.5 * torch.special.erfc(m / math.sqrt(2))
    want = zd.clamp(min=0) - tail
    bound = tail * (2.2e-6 + 9e-8 * m * m) + (want.abs() + tail * 1e-5) * 2.0 ** -24 + 2.0 ** -149
    err = (got - want).abs()
    assert (err <= bound).all(), (err / bound).max()


def test_gelu_of_f16_results(gc):
    # the same bound before the result's own rounding, half a step of f16 (2^-25 at least)
    every = torch.arange(0, 0x8000, device=DEV, dtype=torch.int32).to(torch.int16).view(torch.float16)
    z = every[(every <= 12) & (every > 2.0 ** -10)]
    z = torch.cat([z, -z])
    x = torch.zeros((z.numel(), 16), device=DEV, dtype=torch.float16)
    x[:, 5] = z
    w = torch.zeros((8, 16), device=DEV, dtype=torch.float16)
    w[3, 5] = 1
    got = gc.linear(x, w, activation="gelu")[:, 3].double()
    zd = z.double()
    m = zd.abs()
    tail = m * 0.5 * torch.special.erfc(m / math.sqrt(2))
    want = zd.clamp(min=0) - tail
    before = tail * (2.2e-6 + 9e-8 * m * m) + (want.abs() + tail * 1e-5) * 2.0 ** -24
    bound = before * (1 + 2.0 ** -11) + torch.clamp(want.abs() * 2.0 ** -11, min=2.0 ** -25)
    err = (got - want).abs()
    assert (err <= bound).all(), (err / bound).max()


def test_gelu_far_out(gc):
    inf = float("inf")
    z = torch.tensor([-3e38, -1e5, -40.0, -30.0, -15.0, 15.0, 30.0, 1e5, 3e38, inf, -inf], device=DEV).bfloat16()
    x = torch.zeros((z.numel(), 16), device=DEV, dtype=torch.bfloat16)
    x[:, 0] = z
    w = torch.zeros((4, 16), device=DEV, dtype=torch.bfloat16)
    w[0, 0] = 1
    got = gc.linear(x, w, activation="gelu", out_dtype=torch.float32)[:, 0]
    assert torch.equal(got[5:10], z[5:10].float()) and (got[:5].abs() < 1e-40).all() and got[10] == 0
