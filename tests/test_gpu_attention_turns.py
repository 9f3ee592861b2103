"""Runs of short pieces of two query tiles in one block (heads over 64, whose
products take turns): a piece's first turn comes right behind the last one of
the piece before.  Against the same call with a block for each SM, whose blocks
have one or two pieces each."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


@pytest.mark.parametrize("D", [72, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("lq,lk", [
    ([256] * 40, [100] * 40),                                       # one go a tile
    ([256, 129, 100, 256, 256] * 8, [256, 100, 300, 0, 128] * 8),   # with single tiles and without keys between them
    ([256, 200] * 12, [384, 129] * 12),
], ids=["short", "mixed", "longer"])
def test_runs_of_short_pieces(gc, lq, lk, causal, D):
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda n: torch.randn((n, 2, D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v = r(sum(lq)), r(sum(lk)), r(sum(lk))
    one = gc.attention_plan(lq, lk, 2, 2, D, causal, n_ctas=1)
    wide = gc.attention_plan(lq, lk, 2, 2, D, causal)
    assert one.info.n_joins == 0
    got = [gc.attention(one, q, k, v) for _ in range(3)]
    gc.device_status()
    for x in got[1:]:
        assert torch.equal(x, got[0])
    ref = gc.attention(wide, q, k, v)
    gc.device_status()
    if wide.info.n_joins == 0:
        assert torch.equal(got[0], ref)
    else:  # parts joined: the same but for roundings of the output (2^-8) and of the weights (2^-8 of the values' size)
        assert bool(((got[0].float() - ref.float()).abs() <= 2.0 ** -7 * ref.float().abs() + 2.0 ** -7 * v.float().abs().max()).all())
