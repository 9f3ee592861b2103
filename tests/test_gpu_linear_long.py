"""Matrix products of long summed axes into 16 bits, whose sums are taken in parts.

Whole numbers bit for bit, and products of one sign, where cutting off adds up.  Tolerance: an instruction cuts at most 2^-22 of
the sum so far; over a chain of n that grows evenly that is (n + 1) / 2 * 2^-22 of its sum, with n = 1024 at most
1.23e-4; the parts (of a block, and of a cluster's blocks) are at most 64 + 8, added with 2^-24 each: 4.3e-6.  The result is
looked at through a residual that is nearly its negative, so that its own rounding is of the small difference."""
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


def _whole(shape, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-1, 2, shape, generator=g, device=DEV).float()


# sums stay below 2^24 in any order; few and many tokens, with a part that is not full, one chunk beyond the parts
@pytest.mark.parametrize("dtype", [BF16, F16, E4M3], ids=["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("gated", [False, True], ids=["", "gated"])
@pytest.mark.parametrize("T,K,N", [(1, 16400, 9), (5, 131136, 300), (70, 33024, 700), (33, 32832, 257), (300, 49152, 1500), (1100, 65600, 16),
                                   (9000, 34000, 40), (2600, 40000, 1300), (4100, 16656, 2100)])
def test_whole_numbers(gc, T, K, N, dtype, gated):
    rows = N * (2 if gated else 1)
    x, w = _whole((T, K), T).to(dtype), _whole((rows, K), N).to(dtype)
    od = F16 if dtype is F16 else BF16
    one = dict(x_scale=torch.ones(T, device=DEV), weight_scale=torch.ones(rows, device=DEV)) if dtype is E4M3 else {}
    z = x.float().double() @ w.float().double().T   # (multiples of 1 up to some thousand)
    got = gc.linear(x, w, gated=gated, out_dtype=od, **one)
    if gated:
        # the values times the gates in binary32 may exceed f16: only what fits
        want = (z[:, :N] * z[:, N:]).float().to(od)
    else:
        want = z.float().to(od)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [F16, E4M3], ids=["f16", "e4m3"])
@pytest.mark.parametrize("T,N", [(1300, 1300), (3, 5), (300, 130), (40000, 8)])
@pytest.mark.parametrize("K", [1 << 18, (1 << 20) - 16, 1 << 20])
def test_products_of_one_sign(gc, T, N, K, dtype):
    g = torch.Generator(device=DEV).manual_seed(K)
    x, w = ((torch.rand((1, K), generator=g, device=DEV) + 0.5) for _ in range(2))
    one = {}
    if dtype is E4M3:
        x, w = x.to(dtype), w.to(dtype)
        one = dict(x_scale=torch.full((T,), 1.0 / K, device=DEV), weight_scale=torch.ones(N, device=DEV))
        y = float((x.double() * w.double()).sum()) * float(one["x_scale"][0])
    else:
        x, w = (x / 64).to(dtype), (w * 64 / 1024).to(dtype)
        y = float((x.double() * w.double()).sum())
    near = -torch.full((T, N), y, device=DEV, dtype=torch.float64).to(F16)
    got = gc.linear(x.expand(T, K), w.expand(N, K), residual=near, out_dtype=F16, **one)
    gc.device_status()
    err = (got.double() - near.double() - y).abs().max().item()
    # (the sum before the residual, the residual's addition and the small result's rounding)
    assert err <= y * (1.23e-4 + 4.3e-6 + 2.0 ** -22) + 2.0 ** -11 * abs(y) * 2.0 ** -11 + 2.0 ** -25, err / y
