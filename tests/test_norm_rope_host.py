"""Refusals of geocache_rope_table and geocache_qk_norm_rope (no GPU needed:
arguments are checked before anything is launched)."""
import ctypes

import pytest

from paper_2608_13255_gb300 import build as gbuild


@pytest.fixture(scope="module")
def gc():
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def test_rope_table_checks_arguments(gc):
    L = gc.load()

    def call(rot=64, theta=1e4, scaling=0, factor=1.0, original=0.0, low=1.0, high=32.0, mag=1.0, pos=None, n=16,
             table=4096, row=32, first=0):
        r = gc.Rope(rot, theta, scaling, factor, original, low, high, mag)
        return L.geocache_rope_table(ctypes.byref(r), pos, n, table, row, first, None)

    assert L.geocache_rope_table(None, None, 16, 4096, 32, 0, None) == gc.EINVAL
    for rot in (0, 3, 258, -2):
        assert call(rot=rot) == gc.ESHAPE
    assert call(n=-1) == gc.ESHAPE
    assert call(row=31) == gc.ESHAPE and call(first=1) == gc.ESHAPE and call(first=-1, row=64) == gc.ESHAPE
    assert call(theta=0.0) == gc.EINVAL and call(theta=float("inf")) == gc.EINVAL
    assert call(scaling=4) == gc.EINVAL and call(scaling=-1) == gc.EINVAL
    assert call(scaling=1, factor=0.0) == gc.EINVAL and call(scaling=2, factor=2.0, rot=2) == gc.EINVAL
    assert call(scaling=3, factor=2.0) == gc.EINVAL  # no trained context
    assert call(scaling=3, factor=2.0, original=4096.0, low=32.0, high=32.0) == gc.EINVAL
    assert call(mag=float("nan")) == gc.EINVAL
    assert call(table=None) == gc.EINVAL and call(table=4100) == gc.EINVAL and call(pos=4098) == gc.EINVAL
    assert call(pos=4096 + 64) == gc.EALIAS and "overlaps" in gc.last_error()
    assert gc.last_launches() == 0


def test_norm_rope_checks_arguments(gc):
    L = gc.load()
    T, Hq, Hk, D = 10, 4, 2, 64
    M = 1 << 20

    def heads(data, ts=None, hs=D, H=Hq):
        return gc.Heads(data, H * D if ts is None else ts, hs)

    def call(q=None, k=None, qo=None, ko=None, T=T, Hq=Hq, Hk=Hk, D=D, dtype=1, eps=1e-6, qw=None, table=64 * M, n=100,
             rot=64, layout=0, slots=None):
        q, k = q or heads(M), k or heads(2 * M, H=2)
        qo, ko = qo or heads(3 * M), ko or heads(4 * M, H=2)
        return L.geocache_qk_norm_rope(*map(ctypes.byref, (q, k, qo, ko)), T, Hq, Hk, D, dtype, 1, eps, qw, None, table, n,
                                       rot, layout, slots, None)

    assert call(T=-1) == gc.ESHAPE and call(Hq=-1) == gc.ESHAPE and call(Hk=65537) == gc.ESHAPE
    for d in (0, 4, 60, 264):
        assert call(D=d, rot=0, table=None) == gc.ESHAPE
    assert call(rot=66) == gc.ESHAPE and call(rot=3) == gc.ESHAPE and call(rot=-2) == gc.ESHAPE
    assert call(dtype=3) == gc.EDTYPE
    assert call(layout=2) == gc.EINVAL
    assert call(eps=-1.0) == gc.EINVAL and call(eps=float("nan")) == gc.EINVAL
    assert call(table=None) == gc.EINVAL and call(rot=0) == gc.EINVAL
    assert call(table=64 * M + 4) == gc.EINVAL and call(slots=2 * M + 2) == gc.EINVAL and call(qw=M + 1) == gc.EINVAL
    assert call(n=9) == gc.ESHAPE  # fewer slots than tokens without slots
    assert call(q=heads(None)) == gc.EINVAL and call(qo=heads(M * 3 + 1)) == gc.EINVAL
    assert call(q=heads(M, ts=-1)) == gc.ESHAPE and call(q=heads(M, ts=1 << 39)) == gc.ESHAPE
    # outputs whose rows overlap each other, each other's rows, an input or the table
    assert call(qo=heads(3 * M, ts=0)) == gc.EALIAS and call(qo=heads(3 * M, hs=32)) == gc.EALIAS
    assert call(ko=heads(3 * M + 128, H=2)) == gc.EALIAS
    assert call(qo=heads(M + 128)) == gc.EALIAS and call(qo=heads(2 * M)) == gc.EALIAS
    assert call(ko=heads(64 * M - 64, H=2)) == gc.EALIAS
    assert call(qo=heads(3 * M), slots=3 * M) == gc.EALIAS
    assert gc.last_launches() == 0
    # in place inside one projection's rows of 8 heads the queries and keys do not overlap: what is refused
    # here is a value head written as a query
    row = 8 * D
    q, k = heads(M, ts=row), heads(M + 4 * D * 2, ts=row)
    bad = heads(M + D * 2, ts=row)
    assert call(q=q, k=k, qo=bad, ko=k) == gc.EALIAS
    # heads of q, k and v interleaved: q written into k's place
    q, k = heads(M, ts=12 * D, hs=3 * D), heads(M + 2 * D, ts=12 * D, hs=3 * D)
    assert call(q=q, k=k, Hk=4, qo=heads(M + 2 * D, ts=12 * D, hs=3 * D), ko=heads(4 * M)) == gc.EALIAS


def test_binding_checks_tensors(gc):
    import torch
    q = torch.zeros((4, 2, 64))
    with pytest.raises(ValueError):
        gc.qk_norm_rope(q, q)
    with pytest.raises(TypeError):
        gc.qk_norm_rope(q.double(), q.double())
    with pytest.raises(ValueError):
        gc.rope_table(4, 64, scaling={"kind": "linear", "factor": 2.0, "other": 1})
    with pytest.raises(KeyError):
        gc.rope_table(4, 64, scaling={"kind": "other"})
