"""Outputs that the attention block's calls allocate for a call on another
stream: the memory must be free on that stream, not only on the current one
(where a block that was given back may still have work ahead of it)."""
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


def _behind_pending_work(like, call):
    """call() while a block as large as each of `like` has been given back with a fill of it still ahead on the current
    stream"""
    blocks = [torch.empty_like(x) for x in like]
    torch.cuda._sleep(100_000_000)
    for x in blocks:
        x.fill_(7.0)
    del blocks, x
    got = call()
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("handle", [False, True], ids=["stream", "handle"])
def test_outputs_of_a_call_on_another_stream(gc, handle):
    T, H, D = 700, 4, 64
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v = (torch.randn((T, H, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    plan = gc.attention_plan([T], [T], H, H, D, n_ctas=8)
    st = torch.cuda.Stream()
    at = st.cuda_stream if handle else st
    table = gc.rope_table(T, D)
    qr, kr = gc.qk_norm_rope(q, k, table)
    out = gc.attention(plan, qr, kr, v)
    torch.cuda.synchronize()
    got = _behind_pending_work([table], lambda: gc.rope_table(T, D, stream=at))
    assert torch.equal(got, table)
    got = _behind_pending_work([qr, kr], lambda: gc.qk_norm_rope(q, k, table, stream=at))
    assert torch.equal(got[0], qr) and torch.equal(got[1], kr)
    got = _behind_pending_work([out], lambda: gc.attention(plan, qr, kr, v, stream=at))
    assert torch.equal(got, out)
    # 0 is the legacy default stream
    got = gc.attention(plan, qr, kr, v, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got, out)
    gc.device_status()
