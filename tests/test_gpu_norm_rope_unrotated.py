"""Elements that are not rotated (behind the rotated part of a head, tokens
whose slot is outside the table, calls without a table) do not meet a partner:
a NaN or an infinity among them stays in its own element, or with the norm
reaches the others through the mean alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu

CASES = [(64, 32), (128, 64), (80, 40), (96, 48), (72, 24), (40, 20), (256, 128), (64, 0), (72, 0), (128, 0)]


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _q(D, dtype):
    g = torch.Generator(device="cuda").manual_seed(D)
    return torch.randn((D, 3, D), generator=g, device="cuda").to(dtype)


def _same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("worst", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("D,rot", CASES)
def test_behind_the_rotated_part(gc, D, rot, worst, layout, dtype):
    # token t has its element rot + t % (D - rot) spoiled: every place comes up
    q = _q(D, dtype)
    table = gc.rope_table(D, rot) if rot else None
    at = rot + torch.arange(D, device="cuda") % (D - rot)
    token = torch.arange(D, device="cuda")
    bad = q.clone()
    bad[token, :, at] = worst
    others = torch.ones_like(q, dtype=torch.bool)
    others[token, :, at] = False
    ref, _ = gc.qk_norm_rope(q, None, table, norm=False, layout=layout)
    got, _ = gc.qk_norm_rope(bad, None, table, norm=False, layout=layout)
    assert _same(got[others], ref[others])
    assert _same(got[~others].isnan(), bad[~others].isnan()) and not bool(got[~others].isfinite().any())
    # the mean of the squares is infinite: x * 0 for finite elements
    got, _ = gc.qk_norm_rope(bad, None, table, layout=layout)
    if worst == float("inf"):
        assert bool((got[others] == 0).all()) and bool(got[~others].isnan().all())
    else:
        assert bool(got.isnan().all())
    gc.device_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D", [32, 40, 64, 72, 128, 256])
def test_token_without_a_slot(gc, D, layout, dtype):
    q = _q(D, dtype)
    token = torch.arange(D, device="cuda")
    q[token, :, token] = float("inf")
    slots = torch.full((D,), -1, dtype=torch.int32, device="cuda")
    got, _ = gc.qk_norm_rope(q, None, gc.rope_table(D, D), slots, norm=False, layout=layout)
    with pytest.raises(gc.GeocacheError) as e:
        gc.device_status()
    assert e.value.status == gc.EINVAL
    assert torch.equal(got, q)
