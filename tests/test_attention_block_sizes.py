"""Sizes that the binding of the attention block takes are whole numbers that
fit the C struct: neither cut to an integer nor wrapped to 32 bits."""
import pytest

from paper_2608_13255_gb300 import build as gbuild


@pytest.fixture(scope="module")
def gc():
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


@pytest.mark.parametrize("bad", [dict(Hq=4.5), dict(Hk=2.5), dict(D=64.5), dict(n_ctas=8.5), dict(D=2 ** 32 + 64),
                                 dict(Hq=2 ** 32 + 4), dict(n_ctas=2 ** 32 + 8)], ids=str)
def test_plan_sizes(gc, bad):
    sizes = dict(Hq=4, Hk=2, D=64, n_ctas=8)
    info, _ = gc.plan_attention_host([5], [5], **sizes)
    assert (info.Hq, info.Hk, info.D, info.n_ctas) == (4, 2, 64, 8)
    info, _ = gc.plan_attention_host([5], [5], **{k: float(v) for k, v in sizes.items()})  # whole numbers
    assert info.D == 64
    with pytest.raises((ValueError, gc.GeocacheError)):
        gc.plan_attention_host([5], [5], **{**sizes, **bad})


@pytest.mark.parametrize("bad", [dict(rot=64.5), dict(n_slots=4.5), dict(first_pair=0.5), dict(rot=2 ** 32 + 64),
                                 dict(first_pair=2 ** 32)], ids=str)
def test_rope_table_sizes(gc, bad, monkeypatch):
    # (host memory in the place of a device tensor, and the call itself left out: only the binding is looked at)
    import torch
    called = []
    monkeypatch.setattr(gc, "_dev", lambda t, *a: None if t is None else t.data_ptr())
    monkeypatch.setattr(gc, "_stream", lambda s: None)
    monkeypatch.setattr(gc, "load", lambda: type("L", (), {"geocache_rope_table": lambda *a: called.append(a) or 0}))
    table = torch.empty((4, 32, 2))
    gc.rope_table(4, 64, table=table)
    assert len(called) == 1
    with pytest.raises(ValueError):
        gc.rope_table(**{**dict(n_slots=4, rot=64, table=table), **bad})
    assert len(called) == 1
