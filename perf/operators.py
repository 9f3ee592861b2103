"""The operators of the denoiser's attention block, as measurable cases.

On a cached step only the anchor views go through the denoiser: their rows are packed, keep the rotary slots of the
full view layout, and attend to each other inside their asset.  On a full step all views of an asset attend to each
other.  Two operators carry that: the norms of queries and keys with the rotation of positions (`norm_rope`), and
attention over packed sequences of different lengths (`attention`).

Queries, keys and values are [tokens, heads, D] views of the buffers that their projections write.  A sequence is one
asset (or one prompt); its lengths are given as text, one number for each sequence.  The rotary table, the norms'
weights, the output buffers and the plan of the attention (which depends on the lengths alone) are what a program keeps
over its layers and steps.
"""
import math
import random

import torch

own = False  # False: the plain forms; True: the framework's operators

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------ cases --
def _norm_rope(name, T, n_slots, Hq, Hk, D, rot, dtype="bf16", layout="half", fused=True):
    return dict(name=name, op="norm_rope", T=T, n_slots=n_slots, Hq=Hq, Hk=Hk, D=D, rot=rot, dtype=dtype,
                layout=layout, fused=fused)


def _attention(name, q, k, Hq, Hk, D, dtype="bf16", causal=False, lse=False, fused=True):
    return dict(name=name, op="attention", q=q, k=k, Hq=Hq, Hk=Hk, D=D, dtype=dtype, causal=causal, lse=lse,
                fused=fused)


def listed():
    return [
        # the two anchors of one asset at the 16 x 16 level of a 64 x 64 latent: the smallest call of a cached step
        _norm_rope("norm_rope_anchors_512", T=512, n_slots=1536, Hq=8, Hk=8, D=64, rot=64),
        # all six views of 64 x 64 tokens on a full step
        _norm_rope("norm_rope_full_step_24576", T=24576, n_slots=24576, Hq=16, Hk=16, D=128, rot=128,
                   layout="interleaved"),
        # foreground tokens of one asset in f32, few key heads, half of an 80-wide head rotated
        _norm_rope("norm_rope_ragged_f32", T=5391, n_slots=24576, Hq=20, Hk=4, D=80, rot=40, dtype="f32",
                   fused=False),
        # attention of the two anchors of one asset at the 16 x 16 level: latency counts
        _attention("attn_anchors_512", "512", "512", Hq=8, Hk=8, D=64),
        # two anchors of 64 x 64 tokens: a cached step of one asset
        _attention("attn_anchors_8192", "8192", "8192", Hq=16, Hk=16, D=128),
        # six views of 64 x 64 tokens: a full step of one asset
        _attention("attn_full_step_24576", "24576", "24576", Hq=16, Hk=16, D=128),
        # a batch of assets without their background tokens
        _attention("attn_ragged_assets_f16",
                   "311,7003,1290,4096,2817,905,6144,3333,1777,512,2050,5121,640,4555,1023,3900,2222,129,6500,777,"
                   "3601,1409,2700,5800", "", Hq=12, Hk=12, D=64, dtype="f16"),
        # prompts of different lengths packed, causal, grouped heads
        _attention("attn_causal_packed", "16384,7001,4111,2048,1025,513,64,1", "", Hq=32, Hk=8, D=128, causal=True),
        # the views of four assets read the tokens of their reference images
        _attention("attn_reference_images", "6144,6144,5877,2049", "1370,1370,1370,686", Hq=10, Hk=10, D=80,
                   fused=False),
        # one token for each sequence over what the sequence kept: from a short cache to six views of 64 x 64
        _attention("attn_single_tokens", ",".join(["1"] * 32),
                   "24576,16384,12000,8192,8191,20001,100,4097,6144,9000,15555,2048,3,11111,7000,5000,"
                   "24576,1000,13000,8193,640,18432,10240,777,4096,12288,22222,1,6001,9216,14000,3500",
                   Hq=32, Hk=4, D=128, causal=True, lse=True, fused=False),
        # a few tokens against all six views of 128 x 128: few rows, a long axis, heads of 72
        _attention("attn_few_rows_98304", "17,5", "98304,98303", Hq=16, Hk=16, D=72, lse=True, fused=False),
        # prompts continued after what they kept, rows that see no key, sequences without queries or without keys
        _attention("attn_continued_f16", "700,64,1,0,333,2047", "5200,50,4097,300,0,2047", Hq=12, Hk=2, D=96,
                   dtype="f16", causal=True, lse=True, fused=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.3:
        D = rng.choice([40, 64, 64, 72, 80, 96, 128, 128])
        rot = rng.choice([D, D, D, D // 2])
        Hk = rng.choice([1, 2, 4, 8, 10, 16])
        Hq = Hk * rng.choice([1, 1, 2, 3, 4])
        T = _log(rng, 1, min(49152, 50331648 // ((Hq + Hk) * D)))
        return dict(op="norm_rope", T=T, n_slots=T + rng.randrange(0, 4096), Hq=Hq, Hk=Hk, D=D, rot=rot,
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), layout=rng.choice(["half", "interleaved"]),
                    fused=rng.random() < 0.6)
    D = rng.choice([40, 64, 64, 72, 80, 96, 128, 128, 128])
    Hk = rng.choice([1, 2, 4, 8, 10, 12, 16])
    g = rng.choice([1, 1, 1, 2, 3, 4, 5, 8])
    kind = rng.choice(["self", "self", "self", "cross", "tokens", "continued"])
    n = _log(rng, 1, 48)
    causal = rng.random() < (0.4 if kind == "self" else 0.7 if kind == "continued" else 0.2)
    budget = 4.0e12 / (4.0 * D * Hk * g)  # pairs of a head: the largest listed case costs 4.9e12
    if kind == "self":
        top = max(64, int(min(24576, math.sqrt(budget / n))))
        q = [_log(rng, max(1, top // 32), top) for _ in range(n)]
        k = q
    elif kind == "cross":
        q = [_log(rng, 64, max(65, min(8192, budget / n / 2048))) for _ in range(n)]
        k = [_log(rng, 1, 2048) for _ in range(n)]
    elif kind == "tokens":
        q = [rng.choice([1, 1, 1, 2, 5, 16]) for _ in range(n)]
        k = [_log(rng, 1, min(65536, 4194304 // (n * Hk))) for _ in range(n)]
    else:
        k = [_log(rng, 1, max(64, min(16384, math.sqrt(2 * budget / n)))) for _ in range(n)]
        q = [rng.choice([0, 1, rng.randrange(0, x + 1), rng.randrange(0, x // 2 + 1), min(x + 7, 500)]) for x in k]
        q[0] = max(1, q[0])
    same = kind == "self"
    text = lambda v: ",".join(map(str, v))  # noqa: E731
    return dict(op="attention", q=text(q), k="" if same else text(k), Hq=Hk * g, Hk=Hk, D=D,
                dtype=rng.choice(["bf16", "bf16", "f16"]), causal=causal, lse=rng.random() < 0.5,
                fused=same and rng.random() < 0.7)


def lengths(case):
    q = [int(x) for x in case["q"].split(",")]
    return q, [int(x) for x in case["k"].split(",")] if case["k"] else q


def _pairs(q, k, causal):
    """Visible (query, key) pairs of a sequence: query i sees the keys j <= i + k - q where causal."""
    if not causal:
        return q * k
    n = min(q, k)  # the last n queries see k - n + 1 .. k keys
    return n * (k - n) + n * (n + 1) // 2


def work(case):
    D, Hq, Hk = case["D"], case["Hq"], case["Hk"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm_rope":
        T = case["T"]
        # q and k once in and once out, a table row and a slot for each token, the weights
        rows = min(T, case["n_slots"])
        return {"bytes": 2 * T * (Hq + Hk) * D * e + rows * case["rot"] * 4 + 4 * T + 8 * D,
                "flops": T * (Hq + Hk) * (4 * D + 3 * case["rot"])}
    q, k = lengths(case)
    pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(q, k))
    seen = sum(b for a, b in zip(q, k) if a)  # keys that some query sees
    return {"bytes": 2 * sum(q) * Hq * D * e + 2 * seen * Hk * D * e + (4 * sum(q) * Hq if case["lse"] else 0),
            "flops": 4 * pairs * Hq * D}


# ---------------------------------------------------------------- prepare --
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    D, Hq, Hk = case["D"], case["Hq"], case["Hk"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dt)

    if case["op"] == "norm_rope":
        T, rot = case["T"], case["rot"]
        if case["fused"]:  # one projection wrote queries, keys and values side by side
            qkv = randn(T, Hq + 2 * Hk, D)
            q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        else:
            q, k = randn(T, Hq, D), randn(T, Hk, D)
        freq = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
        angle = torch.arange(case["n_slots"], device=DEV, dtype=torch.float64)[:, None] * freq
        table = torch.stack([angle.cos(), angle.sin()], -1).float()  # [n_slots, rot / 2, 2]
        # the anchors' (or the foreground) tokens in ascending order, each with its slot of the full layout
        slots = torch.randperm(case["n_slots"], generator=gen, device=DEV)[:T].sort().values.to(torch.int32)
        weight = lambda: 1 + 0.1 * torch.randn(D, generator=gen, device=DEV)  # noqa: E731
        return dict(op="norm_rope", q=q, k=k, table=table, slots=slots, q_weight=weight(), k_weight=weight(),
                    layout=case["layout"], eps=1e-6, q_out=torch.empty((T, Hq, D), device=DEV, dtype=dt),
                    k_out=torch.empty((T, Hk, D), device=DEV, dtype=dt))

    lq, lk = lengths(case)
    if case["fused"]:
        qkv = randn(sum(lq), Hq + 2 * Hk, D)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    else:
        q, kv = randn(sum(lq), Hq, D), randn(sum(lk), 2 * Hk, D)
        k, v = kv[:, :Hk], kv[:, Hk:]
    s = dict(op="attention", q=q, k=k, v=v, lq=lq, lk=lk, causal=case["causal"], scale=1.0 / math.sqrt(D),
             out=torch.empty((sum(lq), Hq, D), device=DEV, dtype=dt),
             lse=torch.empty((sum(lq), Hq), device=DEV) if case["lse"] else None)
    if own:
        from paper_2608_13255_gb300 import geocache as gc
        s["plan"] = gc.attention_plan(lq, lk, Hq, Hk, D, causal=case["causal"])
    return s


# -------------------------------------------------------------------- run --
def run(s):
    if own:
        from paper_2608_13255_gb300 import geocache as gc
        if s["op"] == "norm_rope":
            gc.qk_norm_rope(s["q"], s["k"], s["table"], slots=s["slots"], q_weight=s["q_weight"],
                            k_weight=s["k_weight"], eps=s["eps"], layout=s["layout"], q_out=s["q_out"],
                            k_out=s["k_out"])
            return [s["q_out"], s["k_out"]]
        gc.attention(s["plan"], s["q"], s["k"], s["v"], out=s["out"], lse=s["lse"], scale=s["scale"])
        return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]
    if s["op"] == "norm_rope":
        cs = s["table"][s["slots"].long()]
        return [_plain_norm_rope(s["q"], s["q_weight"], cs, s["eps"], s["layout"]),
                _plain_norm_rope(s["k"], s["k_weight"], cs, s["eps"], s["layout"])]
    return _plain_attention(s)


def _plain_norm_rope(x, weight, cs, eps, layout):
    y = x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * weight
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    half = cos.shape[-1]
    if layout == "half":
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, y[..., 2 * half:]], -1).to(x.dtype)


def _plain_attention(s):
    """The sequences have lengths of their own, so each is a product of its own, all heads at once."""
    q, k, v, out, lse = s["q"], s["k"], s["v"], s["out"], s["lse"]
    Hq, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    g, at, bt = Hq // Hk, 0, 0
    for a, b in zip(s["lq"], s["lk"]):
        if a and not b:
            out[at:at + a] = 0
            if lse is not None:
                lse[at:at + a] = -math.inf
        elif a:
            Q = q[at:at + a].float().view(a, Hk, g, D).permute(1, 2, 0, 3).reshape(Hk, g * a, D)
            K = k[bt:bt + b].float().permute(1, 2, 0)
            V = v[bt:bt + b].float().permute(1, 0, 2)
            S = torch.matmul(Q, K).mul_(s["scale"]).view(Hk, g, a, b)
            if s["causal"]:
                i, j = torch.arange(a, device=q.device), torch.arange(b, device=q.device)
                S.masked_fill_(j > i[:, None] + (b - a), -math.inf)
            top = S.amax(-1, keepdim=True).clamp_(min=-3.0e38)  # a row that sees no key has none above it
            S.sub_(top).exp_()
            total = S.sum(-1, keepdim=True)
            O = torch.matmul(S.view(Hk, g * a, b), V).view(Hk, g, a, D)
            O = O / torch.where(total > 0, total, torch.ones_like(total))
            out[at:at + a] = O.permute(2, 0, 1, 3).reshape(a, Hq, D).to(out.dtype)
            if lse is not None:
                lse[at:at + a] = (total.log() + top).squeeze(-1).permute(2, 0, 1).reshape(a, Hq)
        at, bt = at + a, bt + b
    return [out] if lse is None else [out, lse]


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    if work(case)["flops"] > 6e12:  # over about 20 seconds in 64 bits
        return None
    global own
    kept, own = own, False  # the inputs alone
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    f64 = torch.float64
    if s["op"] == "norm_rope":
        half = s["table"].shape[1]
        both = []
        for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            x = x.to(f64)
            y = x / ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]) ** 0.5 * w.to(f64)
            first = torch.arange(half, device=DEV) * (1 if s["layout"] == "half" else 2)
            second = first + (half if s["layout"] == "half" else 1)
            z = torch.view_as_complex(s["table"].to(f64))[s["slots"].long()][:, None]
            turned = torch.complex(y[..., first], y[..., second]) * z
            y[..., first], y[..., second] = turned.real, turned.imag
            both.append(y)
        return both
    Hq, Hk = s["q"].shape[1], s["k"].shape[1]
    out = torch.zeros(s["out"].shape, device=DEV, dtype=f64)
    lse = torch.full(out.shape[:2], -math.inf, device=DEV, dtype=f64)
    at = bt = 0
    for a, b in zip(s["lq"], s["lk"]):
        # rows in blocks that keep the scores under 2 GB
        step = max(1, min(a, (1 << 28) // max(1, b)))
        for h in range(Hq if a and b else 0):
            K, V = s["k"][bt:bt + b, h // (Hq // Hk)].to(f64), s["v"][bt:bt + b, h // (Hq // Hk)].to(f64)
            for r in range(0, a, step):
                n = min(step, a - r)
                S = s["q"][at + r:at + r + n, h].to(f64) @ K.T * s["scale"]
                rows = torch.arange(n, device=DEV)
                if s["causal"]:
                    sees = rows + r + (b - a) + 1
                    S = torch.where(torch.arange(b, device=DEV) < sees[:, None], S, torch.full_like(S, -math.inf))
                    rows = rows[sees > 0]
                S = S[rows]
                z = torch.logsumexp(S, -1)
                lse[at + r + rows, h] = z
                out[at + r + rows, h] = torch.exp(S - z[:, None]) @ V
        at, bt = at + a, bt + b
    return [out] if s["lse"] is None else [out, lse]


if __name__ == "__main__":  # the cases and what each cannot do without
    for c in listed() + [draw(random.Random(i)) for i in range(12)]:
        w = work(c)
        print("%-28s %10.1f MB %10.1f GFLOP  %s" % (c.get("name", "(drawn)"), w["bytes"] / 1e6, w["flops"] / 1e9,
                                                    "" if "name" in c else c))
