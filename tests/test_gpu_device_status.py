"""geocache_device_status gathers what the kernels of all sources have left:
each is reported, by the most telling one where several came together, and all
are cleared by the one read."""
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


def _slot(gc):
    q = torch.zeros((3, 1, 64), device="cuda")
    gc.qk_norm_rope(q, None, gc.rope_table(2, 64), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))


def _wait(gc):
    q = torch.zeros((128, 1, 64), device="cuda", dtype=torch.bfloat16)
    plan = gc.attention_plan([128], [128], 1, 1, 64)
    gc.debug_set_wait(100_000, drop_first_copy=True)
    try:
        gc.attention(plan, q, q, q)
    finally:
        gc.debug_set_wait(0, drop_first_copy=False)


def _face(gc):
    verts = torch.zeros((3, 3), device="cuda")
    faces = torch.tensor([[0, 1, 7]], dtype=torch.int32, device="cuda")
    cams = torch.zeros((1, 1, 16), device="cuda")
    gc.raster_posmaps(verts, faces, torch.tensor([0, 1], dtype=torch.int64, device="cuda"), cams, 8, 8)


def _status(gc, stream=None):
    try:
        gc.device_status(stream)
    except gc.GeocacheError as e:
        return e.status, str(e)
    return gc.OK, ""


@pytest.mark.parametrize("what", [("slot",), ("wait",), ("face",), ("slot", "wait"), ("face", "slot", "wait")], ids="+".join)
def test_every_source_is_read_and_cleared(gc, what):
    assert _status(gc)[0] == gc.OK
    for w in what:
        {"slot": _slot, "wait": _wait, "face": _face}[w](gc)
    launches = gc.last_launches()
    status, text = _status(gc)
    bits = sum({"slot": 32, "wait": 1, "face": 8}[w] for w in what)
    assert "0x%x" % bits in text
    assert status == (gc.ETIMEOUT if what == ("wait",) else gc.EINVAL)
    assert gc.last_launches() == launches  # the status call is not one of the counted ones
    assert _status(gc)[0] == gc.OK


def test_on_another_stream(gc):
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        _slot(gc)
    assert _status(gc, st)[0] == gc.EINVAL and _status(gc, st)[0] == gc.OK
