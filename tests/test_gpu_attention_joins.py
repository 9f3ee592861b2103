"""More joined rows of tiles than a launch with a block for each SM has: a plan
for many more blocks, all of whose units are cut along the keys."""
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


@pytest.mark.parametrize("lq", [1, 37, 128])
def test_many_joins(gc, lq):
    # (outputs within the roundings of the weights and of the output, 2^-8 each, and of binary32 sums, 2^-12)
    H, D, n = 64, 64, 20
    lens_q, lens_k = [lq] * n, [6000 - i for i in range(n)]
    g = torch.Generator(device="cuda").manual_seed(lq)
    r = lambda t: torch.randn((t, H, D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v = r(sum(lens_q)), r(sum(lens_k)), r(sum(lens_k))
    plan = gc.attention_plan(lens_q, lens_k, H, H, D, n_ctas=6000)
    assert plan.info.n_joins > 1024
    plan.workspace.fill_(float("nan"))
    out = gc.attention(plan, q, k, v)
    gc.device_status()
    at = bt = 0
    for a, b in zip(lens_q, lens_k):
        Q, K, V = (x.double().transpose(0, 1) for x in (q[at:at + a], k[bt:bt + b], v[bt:bt + b]))
        P = torch.softmax(Q @ K.transpose(1, 2) * D ** -0.5, -1)
        ref, size = (P @ V).transpose(0, 1), (P @ V.abs()).transpose(0, 1)
        assert bool(((out[at:at + a].double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * (1 + 2.0 ** -8) * ref.abs()).all())
        at, bt = at + a, bt + b
