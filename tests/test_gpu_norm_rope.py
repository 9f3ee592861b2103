"""Norms of queries and keys with the rotation of positions
(geocache_qk_norm_rope) and the rotation's table (geocache_rope_table) against
plain implementations in 64 bits.

Tolerances.  A sum of D <= 256 squares, its mean, root and reciprocal and the
two products that follow are off by less than 2^-20 of the value in binary32;
the rotation adds three roundings of its terms.  So an element is within
2^-19 (|a| + |b|) of the exact one, (a, b) its exact pair before the rotation
(cosines and sines are at most 1 here), plus half a unit of the output's type.
A table entry is within half a binary32 unit (2^-25 of 1) and the rounding of an
angle of up to 10^6 in binary64 (4e-10) of the exact cosine."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF_UNIT = {d: torch.finfo(d).eps / 2 for d in (torch.float32, torch.bfloat16, torch.float16)}  # of a value


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _ref(x, weight, table, slots, rot, layout, eps, norm=True):
    """(exact result, |a| + |b| of each element's pair before the rotation)"""
    y = x.double().cpu()
    if norm:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * weight.double().cpu()
    out, size = y.clone(), y.abs()
    if rot:
        half = rot // 2
        cs = table.double().cpu()[slots.long().cpu()]
        c, s = cs[:, None, :, 0], cs[:, None, :, 1]
        i = torch.arange(half)
        ia, ib = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        a, b = y[..., ia], y[..., ib]
        out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
        size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return out, size


def _check(got, x, weight, table, slots, rot, layout, eps=1e-6, norm=True):
    ref, size = _ref(x, weight, table, slots, rot, layout, eps, norm)
    unit = HALF_UNIT[x.dtype]
    tol = 2.0 ** -19 * size + unit * (ref.abs() + 2.0 ** -19 * size) + 2.0 ** -25
    err = (got.double().cpu() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


def _inputs(gc, T, Hq, Hk, D, rot, dtype, seed=0, n_slots=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((T, Hq, D), generator=g, device="cuda").to(dtype)
    k = (3 * torch.randn((T, Hk, D), generator=g, device="cuda")).to(dtype)
    n = n_slots or 2 * T + 5
    table = gc.rope_table(n, rot) if rot else None
    slots = torch.randint(0, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    w = [1 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2)]
    return q, k, table, slots, w


CASES = [  # T, Hq, Hk, D, rot: every number of lanes a row takes, halves that are whole words and that are not
    (1, 1, 1, 8, 8), (3, 2, 1, 16, 16), (5, 3, 2, 24, 10), (37, 8, 8, 64, 64), (1, 16, 4, 128, 128), (130, 20, 4, 80, 40),
    (7, 5, 5, 72, 72), (33, 12, 3, 96, 48), (9, 4, 1, 256, 256), (11, 3, 7, 160, 64), (6, 9, 2, 200, 2), (40, 40, 1, 40, 36),
    (64, 6, 6, 128, 0),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_matches_64_bit_reference(gc, case, layout, dtype):
    T, Hq, Hk, D, rot = case
    q, k, table, slots, w = _inputs(gc, T, Hq, Hk, D, rot, dtype)
    qo, ko = gc.qk_norm_rope(q, k, table, slots, w[0], w[1], layout=layout)
    assert gc.last_launches() == 1
    _check(qo, q, w[0], table, slots, rot, layout)
    _check(ko, k, w[1], table, slots, rot, layout)
    gc.device_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rot,layout", [(64, "half"), (64, "interleaved"), (20, "half")])
def test_strides_alignment_and_in_place(gc, dtype, rot, layout):
    T, Hq, Hk, D = 45, 6, 2, 64
    _, _, table, slots, w = _inputs(gc, T, Hq, Hk, D, rot, dtype)
    buf = torch.randn((T * (Hq + 2 * Hk) * D + 8,), device="cuda").to(dtype)
    for shift in (0, 1, 4, 8):  # rows on and off 16 and 8 bytes
        qkv = buf[shift:shift + T * (Hq + 2 * Hk) * D].view(T, Hq + 2 * Hk, D).clone() if shift == 0 else \
            buf[shift:shift + T * (Hq + 2 * Hk) * D].view(T, Hq + 2 * Hk, D)
        before = qkv.clone()
        q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        qo, ko = gc.qk_norm_rope(q, k, table, slots, w[0], w[1], layout=layout)
        _check(qo, before[:, :Hq], w[0], table, slots, rot, layout)
        _check(ko, before[:, Hq:Hq + Hk], w[1], table, slots, rot, layout)
        # into head-major outputs
        qh = torch.empty((Hq, T, D), device="cuda", dtype=dtype).transpose(0, 1)
        gc.qk_norm_rope(q, k, table, slots, w[0], w[1], layout=layout, q_out=qh, k_out=ko)
        assert torch.equal(qh, qo)
        # in place inside the projection's output: the values stay as they are
        gc.qk_norm_rope(q, k, table, slots, w[0], w[1], layout=layout, q_out=q, k_out=k)
        assert torch.equal(q, qo) and torch.equal(k, ko)
        assert torch.equal(qkv[:, Hq + Hk:], before[:, Hq + Hk:])


def test_broadcast_heads_and_options(gc):
    T, H, D, rot = 19, 4, 64, 64
    q, k, table, slots, w = _inputs(gc, T, H, 1, D, rot, torch.float32)
    wide = k.expand(T, H, D)  # one head's row read for all heads
    _, ko = gc.qk_norm_rope(q, wide, table, slots, None, w[1])
    _check(ko, wide, w[1], table, slots, rot, "half")
    # no slots: token t has slot t; no keys
    qo, none = gc.qk_norm_rope(q, None, table)
    assert none is None
    _check(qo, q, None, table, torch.arange(T), rot, "half")
    # rotation alone (a weight is then not applied), the norm alone, a large eps
    qo, ko = gc.qk_norm_rope(q, k, table, slots, w[0], w[1], norm=False)
    _check(qo, q, None, table, slots, rot, "half", norm=False)
    qo, _ = gc.qk_norm_rope(q, k, None, None, w[0], w[1], eps=0.5)
    _check(qo, q, w[0], None, None, 0, "half", eps=0.5)
    # a head of zeros stays zero
    z, _ = gc.qk_norm_rope(torch.zeros_like(q), None, table, slots, w[0])
    assert not z.any()


def test_zero_sizes_launch_nothing(gc):
    e = torch.empty((0, 4, 64), device="cuda", dtype=torch.bfloat16)
    gc.qk_norm_rope(e, e, gc.rope_table(4, 64))
    assert gc.last_launches() == 0
    gc.rope_table(0, 64)
    assert gc.last_launches() == 0


def test_slot_out_of_range_is_reported_and_left_unrotated(gc):
    T, H, D = 9, 2, 64
    q, k, table, slots, w = _inputs(gc, T, H, H, D, D, torch.float32, n_slots=12)
    slots[3], slots[7] = -1, 12
    qo, _ = gc.qk_norm_rope(q, k, table, slots, w[0], w[1])
    with pytest.raises(gc.GeocacheError) as e:
        gc.device_status()
    assert e.value.status == gc.EINVAL and "slot" in str(e.value)
    gc.device_status()  # cleared
    good = [t for t in range(T) if t not in (3, 7)]
    _check(qo[good], q[good], w[0], table, slots[good], D, "half")
    _check(qo[[3, 7]], q[[3, 7]], w[0], None, None, 0, "half")


def test_another_stream(gc):
    q, k, table, slots, w = _inputs(gc, 200, 4, 4, 128, 128, torch.bfloat16)
    ref, _ = gc.qk_norm_rope(q, k, table, slots, w[0], w[1])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    out = torch.empty_like(q)
    gc.qk_norm_rope(q, k, table, slots, w[0], w[1], q_out=out, stream=st)
    st.synchronize()
    assert torch.equal(out, ref)


def _frequencies(rot, theta, scaling):
    i = np.arange(rot // 2)
    kind, f = scaling.get("kind", "plain"), scaling.get("factor", 1.0)
    if kind == "base":
        theta = theta * f ** (rot / (rot - 2))
    fr = theta ** (-2.0 * i / rot)
    if kind == "linear":
        fr = fr / f
    if kind == "by_parts":
        turns = scaling["original"] * fr / (2 * math.pi)
        lo, hi = scaling.get("low", 1.0), scaling.get("high", 32.0)
        r = np.clip((turns - lo) / (hi - lo), 0, 1)
        fr = fr * (r + (1 - r) / f)
    return fr


@pytest.mark.parametrize("scaling", [{}, {"kind": "linear", "factor": 4.0}, {"kind": "base", "factor": 8.0},
                                     {"kind": "by_parts", "factor": 4.0, "original": 4096}],
                         ids=lambda s: s.get("kind", "plain"))
@pytest.mark.parametrize("rot,theta", [(64, 10000.0), (128, 500000.0), (6, 100.0)])
def test_table(gc, rot, theta, scaling):
    n = 777
    pos = (torch.arange(n, dtype=torch.int32) * 1283 - 500).cuda()
    got = gc.rope_table(rot=rot, theta=theta, pos=pos, scaling=scaling, magnitude=1.25).cpu().double().numpy()
    ang = pos.cpu().double().numpy()[:, None] * _frequencies(rot, theta, scaling)
    tol = 1.25 * (2.0 ** -24 + 1e-9)
    assert np.abs(got[..., 0] - 1.25 * np.cos(ang)).max() <= tol
    assert np.abs(got[..., 1] - 1.25 * np.sin(ang)).max() <= tol
    plain = gc.rope_table(n, rot, theta, scaling=scaling).cpu().double().numpy()
    ang = np.arange(n)[:, None] * _frequencies(rot, theta, scaling)
    assert np.abs(plain[..., 0] - np.cos(ang)).max() <= 2.0 ** -24 + 1e-9


def test_table_of_two_axes(gc):
    # rows and columns of an 8 x 6 token grid, half of the pairs each
    H, W, rot = 8, 6, 32
    y = torch.arange(H * W, dtype=torch.int32) // W
    x = torch.arange(H * W, dtype=torch.int32) % W
    table = torch.full((H * W, rot, 2), 7.0, device="cuda")
    gc.rope_table(rot=rot, pos=y.cuda(), table=table)
    assert bool((table[:, rot // 2:] == 7.0).all())  # pairs of the other axis untouched
    gc.rope_table(rot=rot, pos=x.cuda(), table=table, first_pair=rot // 2)
    fr = _frequencies(rot, 10000.0, {})
    for a, p in ((0, y), (rot // 2, x)):
        got = table[:, a:a + rot // 2].cpu().double().numpy()
        ang = p.double().numpy()[:, None] * fr
        assert np.abs(got[..., 0] - np.cos(ang)).max() <= 2.0 ** -24 + 1e-9
        assert np.abs(got[..., 1] - np.sin(ang)).max() <= 2.0 ** -24 + 1e-9
