"""The running rescale of the attention: scores that climb along the keys, so
that rows take a new maximum several times inside one piece while their
neighbours in the warp do not, and the keys before each change still carry
weight (a wrong factor, a column of the output or a sum that is left behind
shows).  In one piece, and in parts that are joined.

Tolerance.  A score is a binary32 sum of D exact products: off by at most
D 2^-23 S, S the largest scale sum_d |q_d k_d|.  The exponent's two roundings
and the exponential add less than 2^-17 for the scores here (below 2^6).  With
e the sum of the two, weights and their sum are within e of themselves each;
a weight is rounded to the inputs' type (u of itself) for the product, whose n
terms are summed in binary32 (n 2^-23).  So
    |out - exact| <= (u + 2 e + n 2^-23) A + u (1 + 2^-6) |exact|,
A = sum_j p_j |v_j|, and lse is within 2 e + n 2^-24 and 2^-22 of itself.  f16
weights below 2^-14 of the row's reference are off by up to 2^-25 of it instead:
n 2^-25 max |v| more."""
import math

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


GAINS = (1.0, 0.0, 0.5, -1.0)  # of the climb, by row: neighbours in a warp differ


def _inputs(lq, lk, H, D, dtype, device="cuda"):
    """Keys whose scores for gain 1 climb by 5.2 and 1.1 in turns from tile to tile: 128 exp(5.2) stays below 2^15, the
    sum behind the next 1.1 does not."""
    g = torch.Generator(device=device).manual_seed(D)
    r = lambda n: torch.randn((n, H, D), generator=g, device=device)  # noqa: E731
    tile = torch.arange(lk, device=device) // 128
    level = (tile // 2) * 6.3 + (tile % 2) * 5.2
    side = torch.where(torch.arange(D, device=device) % 3 == 0, -1.0, 1.0)
    gain = torch.tensor(GAINS, device=device)[torch.arange(lq, device=device) % 4]
    q = gain[:, None, None] * side + 0.05 * r(lq)
    k = level[:, None, None] / D ** 0.5 * side + 0.1 * r(lk)
    return q.to(dtype), k.to(dtype), r(lk).to(dtype)


def _scores(q, k, causal):
    lq, lk, D = q.shape[0], k.shape[0], q.shape[2]
    S = q.double().transpose(0, 1) @ k.double().permute(1, 2, 0) * D ** -0.5
    if causal:
        i, j = torch.arange(lq, device=q.device), torch.arange(lk, device=q.device)
        S = S.masked_fill(j > i[:, None] + (lk - lq), -math.inf)
    return S


def _rescales(S):
    """Times each row [H, lq] takes a new maximum in one piece."""
    m = S[..., :128].amax(-1)
    n = torch.zeros_like(m)
    for a in range(128, S.shape[-1], 128):
        t = S[..., a:a + 128]
        new = torch.exp(t - m[..., None]).sum(-1) > 2.0 ** 15
        n += new
        m = torch.where(new, torch.maximum(m, t.amax(-1)), m)
    return n


def _check(out, lse, q, k, v, causal):
    D, n, u = q.shape[2], k.shape[0], torch.finfo(q.dtype).eps / 2
    S = _scores(q, k, causal)
    z = torch.logsumexp(S, -1)
    P, V = torch.exp(S - z[..., None]), v.double().transpose(0, 1)
    ref, size = (P @ V).transpose(0, 1), (P @ V.abs()).transpose(0, 1)
    top = float((q.double().abs().transpose(0, 1) @ k.double().abs().permute(1, 2, 0)).max()) * D ** -0.5
    e = D * 2.0 ** -23 * top + 2.0 ** -17
    tol = (u + 2 * e + n * 2.0 ** -23) * size + u * (1 + 2.0 ** -6) * ref.abs()
    if q.dtype is torch.float16:
        tol = tol + n * 2.0 ** -25 * float(v.double().abs().max()) + 2.0 ** -25
    err = (out.double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    z = z.transpose(0, 1)
    assert bool(((lse.double() - z).abs() <= 2 * e + n * 2.0 ** -24 + 2.0 ** -22 * z.abs()).all())


@pytest.mark.parametrize("D", [8, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("lq,n_ctas", [(300, 1), (150, 3)], ids=["whole", "joined"])
def test_new_maxima_along_the_keys(gc, lq, n_ctas, causal, dtype, D):
    H, lk = 2, 128 * 14 + 100
    q, k, v = _inputs(lq, lk, H, D, dtype)
    plan = gc.attention_plan([lq], [lk], H, H, D, causal, n_ctas=n_ctas)
    n = _rescales(_scores(q, k, causal))
    for i, gain in enumerate(GAINS):
        rows = n[:, i::4]
        assert bool((rows >= 3).all()) if gain == 1.0 else gain == 0.5 or not bool(rows.any())
    info, schedule = gc.plan_attention_host([lq], [lk], H, H, D, causal, n_ctas)
    at = (info.n_ctas + 1 + 15) // 16 * 16
    tiles = schedule.numpy()[at:at + 16 * info.n_items].reshape(-1, 16)[:, 8:10].max(1)
    if n_ctas == 1:
        assert info.n_joins == 0 and tiles.max() == 15
    else:
        assert info.n_joins > 0 and (tiles >= 5).sum() >= 2  # the climb goes on inside a part
    out = torch.full_like(q, float("nan"))
    lse = torch.full((lq, H), float("nan"), device="cuda")
    gc.attention(plan, q, k, v, out=out, lse=lse)
    gc.device_status()
    _check(out, lse, q, k, v, causal)
