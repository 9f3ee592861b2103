"""qk_norm_rope and rope_table inside a captured graph: the replay reads what
its inputs hold then."""
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


@pytest.mark.parametrize("D,rot,dtype", [(64, 64, torch.bfloat16), (80, 40, torch.float16), (40, 20, torch.float32)])
def test_replay(gc, D, rot, dtype):
    T, Hq, Hk = 130, 6, 2
    g = torch.Generator(device="cuda").manual_seed(D)
    new = lambda: torch.randn((T, Hq + 2 * Hk, D), generator=g, device="cuda").to(dtype)  # noqa: E731
    qkv, other = new(), new()
    pos = torch.randint(0, 4096, (T,), generator=g, device="cuda", dtype=torch.int32)
    slots = torch.randperm(T, generator=g, device="cuda").to(torch.int32)
    table = torch.empty((T, rot // 2, 2), device="cuda")
    q_out, k_out = torch.empty((T, Hq, D), dtype=dtype, device="cuda"), torch.empty((T, Hk, D), dtype=dtype, device="cuda")

    def call():
        gc.rope_table(rot=rot, pos=pos, table=table)
        gc.qk_norm_rope(qkv[:, :Hq], qkv[:, Hq:Hq + Hk], table, slots, q_out=q_out, k_out=k_out)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for values in (other, new()):
        qkv.copy_(values)
        pos.add_(7)
        graph.replay()
        got = q_out.clone(), k_out.clone(), table.clone()
        for x in (q_out, k_out, table):
            x.fill_(float("nan"))
        call()
        for x, y in zip(got, (q_out, k_out, table)):
            assert torch.equal(x, y)
    gc.device_status()
