"""Rows that see no key, beside values that are not finite: the definition
gives 0 and -inf for them, whatever lies behind the mask."""
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


@pytest.mark.parametrize("D", [40, 64, 72, 128])
@pytest.mark.parametrize("worst", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("Hq,n_ctas", [(2, 0), (2, 1), (8, 0)])
def test_empty_rows_beside_values_that_are_not_finite(gc, worst, D, Hq, n_ctas):
    # causal: of 300 queries on 100 keys the first 200 see none, and share a tile with rows that do
    lq, lk, empty, at = [300, 70], [100, 70], 200, 5
    g = torch.Generator(device="cuda").manual_seed(6)
    r = lambda n, h: torch.randn((n, h, D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v = r(sum(lq), Hq), r(sum(lk), 2), r(sum(lk), 2)
    plan = gc.attention_plan(lq, lk, Hq, 2, D, causal=True, n_ctas=n_ctas)
    ref = gc.attention(plan, q, k, v).clone()
    v[at] = worst
    lse = torch.full((sum(lq), Hq), float("nan"), device="cuda")
    got = gc.attention(plan, q, k, v, lse=lse)
    gc.device_status()
    assert not bool(got[:empty].any())  # zeros, no NaN
    assert bool((lse[:empty] == -float("inf")).all()) and bool(torch.isfinite(lse[empty:]).all())
    assert not bool(torch.isfinite(got[empty + at:lq[0]]).any())  # these see it
    assert torch.equal(got[lq[0]:], ref[lq[0]:])                  # another sequence
