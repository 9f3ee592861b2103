"""Attention whose bounded waits run out while copies and products are in
flight: the blocks that give up end without leaving a copy behind that could
land in the shared memory of the next one.  What must not happen cannot be
observed without a race, so these tests check the surroundings of it: the
timeout is reported, the launch queued directly behind gives the same bits as
ever, and a run that does not give up reports nothing."""
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


def _inputs(lq, lk, H, D, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda n: torch.randn((n, H, D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    return r(sum(lq)), r(sum(lk)), r(sum(lk))


def _under_a_limit(gc, call):
    """`call` under a limit, the same call directly behind it under the default one: (outputs of both, whether a wait
    ran out)"""
    try:
        first = call()
        gc.debug_set_wait(0, drop_first_copy=False)
        second = call()  # queued behind, before anything is waited for
        torch.cuda.synchronize()
        late = False
        try:
            gc.device_status()
        except gc.GeocacheError as e:
            assert e.status == gc.ETIMEOUT
            late = True
    finally:
        gc.debug_set_wait(0, drop_first_copy=False)
    gc.device_status()
    return first, second, late


@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("n_ctas", [1, 152])
def test_limit_shorter_than_a_copy(gc, D, n_ctas):
    # 1 ns: a block gives up at its first wait that does not end by itself, with a ring of copies on its way.  (One try of
    # a wait lets the thread sleep for as long as the hardware likes, so a block may get through; its results are then
    # whole.)
    lq, lk = [300, 1, 512], [2000, 700, 512]
    q, k, v = _inputs(lq, lk, 2, D)
    plan = gc.attention_plan(lq, lk, 2, 2, D, n_ctas=n_ctas)
    ref = gc.attention(plan, q, k, v).clone()
    gc.device_status()
    for _ in range(5):
        gc.debug_set_wait(1, drop_first_copy=False)
        first, second, late = _under_a_limit(gc, lambda: gc.attention(plan, q, k, v))
        assert late or torch.equal(first, ref)
        assert torch.equal(second, ref)


@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("n_tiles", [1, 2, 3, 4, 5, 6, 9])
def test_first_copy_left_out(gc, D, n_tiles):
    # pieces shorter and longer than the ring (of 8 stages, 5 for heads over 64): the loads end before a wait runs out, or
    # wait for a stage themselves
    lq, lk = [256, 256], [128 * n_tiles, 128 * n_tiles]
    q, k, v = _inputs(lq, lk, 2, D, seed=n_tiles)
    plan = gc.attention_plan(lq, lk, 2, 2, D, n_ctas=1)
    ref = gc.attention(plan, q, k, v).clone()
    gc.device_status()
    gc.debug_set_wait(200_000, drop_first_copy=True)
    _, second, late = _under_a_limit(gc, lambda: gc.attention(plan, q, k, v))
    assert late and torch.equal(second, ref)
