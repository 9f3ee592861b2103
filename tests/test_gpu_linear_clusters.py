"""Matrix products whose summed axis is cut over a cluster, when a wait runs out: every block still sends the others all of
their sums and waits for its own, so that none ends with some on their way to it.  Calls queued directly behind, which take
the same shared memory, give the results that they give alone, and the status says what happened."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _operands(gc, T, K, N, dtype, gated):
    g = torch.Generator(device=DEV).manual_seed(T + K + N)
    x = torch.randn((T, K), generator=g, device=DEV)
    w = torch.randn((N * (2 if gated else 1), K), generator=g, device=DEV) * K ** -0.5
    if dtype is BF16:
        return dict(x=x.to(dtype), weight=w.to(dtype), gated=gated)
    (x, xs), (w, ws) = gc.quantize_rows(x), gc.quantize_rows(w)
    return dict(x=x, weight=w, x_scale=xs, weight_scale=ws, gated=gated)


@pytest.mark.parametrize("T,K,N,dtype,od,gated", [(4, 4096, 512, BF16, BF16, False), (1, 10240, 300, E4M3, F32, False),
                                                  (81, 6096, 1831, BF16, BF16, False), (40, 8192, 700, BF16, F32, True),
                                                  (265, 11744, 932, E4M3, F32, True)],
                         ids=lambda v: str(v).replace("torch.", ""))
def test_sums_on_their_way(gc, T, K, N, dtype, od, gated):
    a = _operands(gc, T, K, N, dtype, gated)
    other = _operands(gc, 16, 512, 1024, BF16, False)
    want, want_other = gc.linear(out_dtype=od, **a), gc.linear(**other)
    gc.device_status()
    for limit, drop in ((100_000, True), (1, True), (1, False)):
        late = 0
        try:
            for _ in range(10):
                gc.debug_set_wait(limit, drop_first_copy=drop)
                gc.linear(out_dtype=od, **a)
                gc.debug_set_wait(0, drop_first_copy=False)
                behind = [gc.linear(**other), gc.linear(out_dtype=od, **a), gc.linear(**other)]
                torch.cuda.synchronize()
                try:
                    gc.device_status()
                except gc.GeocacheError as e:
                    assert e.status == gc.ETIMEOUT
                    late += 1
                assert torch.equal(behind[0], want_other) and torch.equal(behind[1], want) and torch.equal(behind[2], want_other)
        finally:
            gc.debug_set_wait(0, drop_first_copy=False)
        assert late == 10 or not drop
    gc.device_status()
