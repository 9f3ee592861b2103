"""Attention over packed sequences (geocache_attention) against a plain
implementation in 64 bits.

Tolerance.  A weight exp(...) is rounded to the inputs' type (half a unit u of
itself: 2^-8 of it for bf16, 2^-11 for f16) while the sum is not, so an output
is within u * sum_j p_j |v_j| of the exact one before it is rounded to the type
itself.  Scores are binary32 sums of exact products: off by at most
D 2^-24 sum_d |q_d k_d| scale <= 2^-14 here, and the exponential adds 2^-21, which
changes a weight by less than 2^-13 of itself.  So |out - exact| <= (u + 2^-12) A
+ u |exact| (1 + u) with A = sum_j p_j |v_j|, and lse is within 2^-13 (and 2^-22 of itself).
f16 weights below 2^-14 lose relative accuracy: at most 2^-25 each of the row's
largest, which adds n 2^-25 max |v| for n keys."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {d: torch.finfo(d).eps / 2 for d in (torch.bfloat16, torch.float16)}


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13255_gb300 import build as gbuild
    gbuild.build()
    from paper_2608_13255_gb300 import geocache
    geocache.load()
    return geocache


def _exact(q, k, v, lq, lk, causal, scale):
    """(out, A, lse) in 64 bits on the device"""
    Hq, Hk = q.shape[1], k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(out)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    at = bt = 0
    for a, b in zip(lq, lk):
        if a and b:
            Q = q[at:at + a].double().transpose(0, 1)
            K = k[bt:bt + b].double().transpose(0, 1).repeat_interleave(Hq // Hk, 0)
            V = v[bt:bt + b].double().transpose(0, 1).repeat_interleave(Hq // Hk, 0)
            S = Q @ K.transpose(1, 2) * scale
            if causal:
                i, j = torch.arange(a, device=q.device), torch.arange(b, device=q.device)
                S = S.masked_fill(j > i[:, None] + (b - a), -math.inf)
            z = torch.logsumexp(S, -1)
            P = torch.where(torch.isinf(z)[..., None], torch.zeros_like(S), torch.exp(S - z[..., None]))
            out[at:at + a] = (P @ V).transpose(0, 1)
            size[at:at + a] = (P @ V.abs()).transpose(0, 1)
            lse[at:at + a] = z.transpose(0, 1)
        at, bt = at + a, bt + b
    return out, size, lse


def _check(got, lse, q, k, v, lq, lk, causal, scale):
    ref, size, z = _exact(q, k, v, lq, lk, causal, scale)
    u = U[q.dtype]
    tol = (u + 2.0 ** -12) * size + u * (1 + u) * ref.abs()
    if q.dtype is torch.float16:
        tol = tol + max(lk) * 2.0 ** -25 * (v.abs().max().double() if v.numel() else 0) + 2.0 ** -25
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), float((err - tol)[bad].max()))
    if lse is not None:
        fin = torch.isfinite(z)
        assert torch.equal(torch.isfinite(lse), fin) and bool((lse[~fin] == -math.inf).all())
        assert bool(((lse.double() - z).abs()[fin] <= 2.0 ** -13 + 2.0 ** -22 * z.abs()[fin]).all())


def _inputs(lq, lk, Hq, Hk, D, dtype, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda n, h: torch.randn((n, h, D), generator=g, device="cuda")  # noqa: E731
    return (spread * r(sum(lq), Hq)).to(dtype), r(sum(lk), Hk).to(dtype), r(sum(lk), Hk).to(dtype)


def _run(gc, lq, lk, Hq, Hk, D, causal, dtype, seed=0, spread=1.0, n_ctas=0, scale=None):
    q, k, v = _inputs(lq, lk, Hq, Hk, D, dtype, seed, spread)
    plan = gc.attention_plan(lq, lk, Hq, Hk, D, causal, n_ctas=n_ctas)
    if plan.workspace is not None:
        plan.workspace.fill_(float("nan"))  # its contents need not be set
    out = torch.full((sum(lq), Hq, D), float("nan"), dtype=dtype, device="cuda")
    lse = torch.full((sum(lq), Hq), float("nan"), device="cuda")
    gc.attention(plan, q, k, v, out=out, lse=lse, scale=scale)
    if sum(lq):
        assert gc.last_launches() == (2 if plan.info.n_joins else 1)
    _check(out, lse, q, k, v, lq, lk, causal, D ** -0.5 if scale is None else scale)
    gc.device_status()
    return plan


@pytest.mark.parametrize("D", [8, 16, 40, 64, 72, 80, 96, 120, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_head_sizes(gc, D, dtype):
    _run(gc, [200, 130], [300, 257], 4, 2, D, False, dtype)
    _run(gc, [200, 130], [300, 257], 4, 2, D, True, dtype)


LENGTHS = [
    ([1], [1]), ([1], [128]), ([1], [129]), ([128], [127]), ([129], [128]), ([255], [256]), ([257], [1]),
    ([1, 1, 1], [1000, 16, 17]), ([0, 3, 0], [5, 0, 7]), ([512], [512]), ([300], [40]), ([2, 500, 64, 1], [700, 20, 64, 1]),
    ([1], [20000]), ([33, 5], [6000, 5999]),
]


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("lq,lk", LENGTHS, ids=str)
def test_lengths(gc, lq, lk, causal):
    _run(gc, lq, lk, 2, 2, 64, causal, torch.bfloat16)
    _run(gc, lq, lk, 3, 1, 128, causal, torch.float16)


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (5, 5), (6, 2), (7, 1), (8, 1), (40, 8), (24, 2), (128, 1), (130, 1), (96, 2)])
def test_grouped_heads(gc, Hq, Hk):
    for causal in (False, True):
        _run(gc, [70, 1, 150], [300, 513, 150], Hq, Hk, 64, causal, torch.bfloat16)


@pytest.mark.parametrize("n_ctas", [1, 5, 37, 152])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_division_of_the_work(gc, n_ctas, causal):
    # the same work as whole tiles and cut along the keys: many parts a row, and parts that some rows do not see
    plan = _run(gc, [260, 17, 128], [2600, 1111, 128], 2, 1, 128, causal, torch.bfloat16, n_ctas=n_ctas)
    if n_ctas in (1, 152):  # between them the plan may do either
        assert (plan.info.n_joins > 0) == (n_ctas == 152)
    _run(gc, [260, 17, 128], [2600, 1111, 128], 2, 1, 64, causal, torch.float16, n_ctas=n_ctas)


@pytest.mark.parametrize("D", [8, 24, 80])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_pairs_of_tiles_beside_single_ones(gc, D, causal):
    # one block takes pairs of query tiles, single tiles, tiles that see fewer keys than their neighbour and none at all,
    # one after the other: each warp has to keep its place in the ring of stages through what only the other tile reads
    lq = [1, 300, 5, 256, 64, 400, 1, 130, 700, 3]
    lk = [900, 300, 1500, 40, 700, 0, 1, 2000, 650, 129]
    _run(gc, lq, lk, 3, 3, D, causal, torch.bfloat16, n_ctas=1)
    _run(gc, lq, lk, 2, 1, D, causal, torch.float16, n_ctas=2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_peaked_and_growing_scores(gc, dtype):
    # scores whose maximum grows along the keys (the running rescale) and spreads over many powers of two
    lq, lk, H, D = [150], [900], 2, 64
    q, k, v = _inputs(lq, lk, H, H, D, dtype, seed=3)
    ramp = torch.linspace(0.1, 6.0, lk[0], device="cuda")[:, None, None]
    q = q.abs()
    k = (k.abs().float() * ramp / 6).to(dtype)
    for order in (k, k.flip(0)):
        plan = gc.attention_plan(lq, lk, H, H, D)
        out, lse = torch.empty_like(q), torch.empty((lq[0], H), device="cuda")
        gc.attention(plan, q, order, v, out=out, lse=lse, scale=0.5)
        # (scores reach 30 and their rounding D 2^-24 sum |q k| scale 2^-18: still inside the tolerance)
        _check(out, lse, q, order, v, lq, lk, False, 0.5)


def test_scale(gc):
    _run(gc, [100], [200], 2, 2, 64, False, torch.bfloat16, scale=1.0 / 64)
    _run(gc, [100], [200], 2, 2, 64, True, torch.bfloat16, scale=1e-4)


def test_views_of_one_projection(gc):
    lens, Hq, Hk, D = [200, 1, 333], 6, 2, 72
    T = sum(lens)
    qkv = torch.randn((T, Hq + 2 * Hk, D), device="cuda", dtype=torch.float32).to(torch.bfloat16)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    plan = gc.attention_plan(lens, lens, Hq, Hk, D, True)
    ref = gc.attention(plan, q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(gc.attention(plan, q, k, v), ref)
    _check(ref, None, q, k, v, lens, lens, True, D ** -0.5)
    # head-major tensors, and an output inside a wider buffer whose other rows stay
    hm = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    wide = torch.full((T, Hq + 1, D), 7.0, device="cuda", dtype=torch.bfloat16)
    gc.attention(plan, hm(q), hm(k), hm(v), out=wide[:, :Hq])
    assert torch.equal(wide[:, :Hq], ref) and bool((wide[:, Hq] == 7.0).all())


def test_broadcast_tensors(gc):
    # one head's keys and values for all heads, one query for all tokens: strides of zero
    T, H, D = 70, 3, 64
    q, k, v = _inputs([T], [T], H, 1, D, torch.bfloat16)
    wide_k, wide_v = k.expand(T, H, D), v.expand(T, H, D)
    plan = gc.attention_plan([T], [T], H, H, D)
    ref = gc.attention(plan, q, wide_k.contiguous(), wide_v.contiguous())
    assert torch.equal(gc.attention(plan, q, wide_k, wide_v), ref)
    one = q[:1].expand(T, H, D)
    assert torch.equal(gc.attention(plan, one, wide_k, wide_v), gc.attention(plan, one.contiguous(), wide_k, wide_v))


def test_same_bits_in_every_call_and_on_another_stream(gc):
    lq, lk = [17, 300], [5000, 2500]
    q, k, v = _inputs(lq, lk, 4, 2, 128, torch.bfloat16)
    plan = gc.attention_plan(lq, lk, 4, 2, 128)
    assert plan.info.n_joins
    ref = gc.attention(plan, q, k, v)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    ws = torch.empty_like(plan.workspace)
    out = torch.empty_like(ref)
    gc.attention(plan, q, k, v, out=out, workspace=ws, stream=st)
    for _ in range(3):
        assert torch.equal(gc.attention(plan, q, k, v), ref)
    st.synchronize()
    assert torch.equal(out, ref)


def test_graph_capture(gc):
    lq, lk = [64, 1], [3000, 70]
    q, k, v = _inputs(lq, lk, 4, 4, 64, torch.bfloat16)
    plan = gc.attention_plan(lq, lk, 4, 4, 64)
    ref = gc.attention(plan, q, k, v)
    out = torch.empty_like(ref)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gc.attention(plan, q, k, v, out=out)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("worst", [float("nan"), float("inf"), -float("inf")], ids=str)
def test_a_sequence_does_not_read_its_neighbours(gc, worst, D):
    # NaN and infinities in the sequences before and behind, whose rows lie in the same tiles
    lens = [70, 201, 90]
    q, k, v = _inputs(lens, lens, 2, 2, D, torch.bfloat16)
    plan = gc.attention_plan(lens, lens, 2, 2, D)
    ref = gc.attention(plan, q, k, v)
    rows = torch.ones(sum(lens), dtype=torch.bool, device="cuda")
    rows[70:271] = False
    for x in (q, k, v):
        x[rows] = worst
    got = gc.attention(plan, q, k, v)
    assert torch.equal(got[70:271], ref[70:271])


def test_not_a_number_stays_in_its_rows(gc):
    lens = [300]
    q, k, v = _inputs(lens, lens, 1, 1, 64, torch.bfloat16)
    plan = gc.attention_plan(lens, lens, 1, 1, 64, causal=True)
    ref = gc.attention(plan, q, k, v)
    q[17] = float("nan")
    k[250] = float("nan")  # seen by the rows from 250 on
    got = gc.attention(plan, q, k, v)
    assert bool(torch.isnan(got[17]).all()) and bool(torch.isnan(got[250:]).all())
    keep = [i for i in range(250) if i != 17]
    assert torch.equal(got[keep], ref[keep])


def test_wait_that_runs_out_is_reported_and_the_context_stays_usable(gc):
    lens = [512]
    q, k, v = _inputs(lens, lens, 8, 8, 64, torch.bfloat16)
    plan = gc.attention_plan(lens, lens, 8, 8, 64)
    ref = gc.attention(plan, q, k, v)
    gc.device_status()
    gc.debug_set_wait(200_000, drop_first_copy=True)  # the first block's first keys are never copied
    try:
        gc.attention(plan, q, k, v)
        torch.cuda.synchronize()
        with pytest.raises(gc.GeocacheError) as e:
            gc.device_status()
        assert e.value.status == gc.ETIMEOUT
        gc.device_status()
    finally:
        gc.debug_set_wait(0, drop_first_copy=False)
    assert torch.equal(gc.attention(plan, q, k, v), ref)
    gc.device_status()


def test_sequences_beyond_32_bit_offsets(gc):
    # keys whose elements lie past 2^32: the last sequence of a long packed cache
    Hk, D = 8, 128
    lk = [2_200_000, 3000]
    kv = torch.empty((sum(lk), 2 * Hk, D), device="cuda", dtype=torch.bfloat16)
    assert kv.numel() > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(1)
    tail = torch.randn((lk[1], 2 * Hk, D), generator=g, device="cuda").to(torch.bfloat16)
    kv[:lk[0]] = 1.0
    kv[lk[0]:] = tail
    lq = [0, 9]
    q = torch.randn((9, Hk, D), generator=g, device="cuda").to(torch.bfloat16)
    plan = gc.attention_plan(lq, lk, Hk, Hk, D)
    got = gc.attention(plan, q, kv[:, :Hk], kv[:, Hk:])
    _check(got, None, q, tail[:, :Hk], tail[:, Hk:], [9], [lk[1]], False, D ** -0.5)
