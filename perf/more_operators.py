"""The operators around the attention in a denoiser's block, as measurable cases.

A block of the anchor-only forward is: residual + norm, projection to queries, keys and values, attention, projection
back into the residual; residual + norm, feed-forward (up with an activation, down into the residual).  Three operators
carry what is not attention: the norm with the residual's addition and an output in the inputs' type or in 8 bits with a
scale for each row (`add_rms_norm`), the same 8-bit form of rows that follow no norm (`quantize_rows`), and the matrix
product with bias, activation and residual in its epilogue (`linear`), on 16-bit operands or on 8-bit ones with scales.

Rows are tokens: those of the views that take part, of all assets, one after the other.  Output buffers are what a
program keeps over its layers and steps; weights in 8 bits are made once, when a model is loaded.
"""
import math
import random

import torch

own = False  # False: the plain forms; True: the framework's operators

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
E4M3_MAX = 448.0
TINY = 2.0 ** -126  # the least scale


# ------------------------------------------------------------------ cases --
def _norm(name, T, C, dtype="bf16", residual="bf16", out="e4m3", strided=False):
    return dict(name=name, op="add_rms_norm", T=T, C=C, dtype=dtype, residual=residual, out=out, strided=strided)


def _quantize(name, T, C, dtype="bf16", strided=False):
    return dict(name=name, op="quantize_rows", T=T, C=C, dtype=dtype, strided=strided)


def _linear(name, T, K, N, dtype="bf16", out="bf16", bias=True, act="", gated=False, residual=False, strided=False):
    return dict(name=name, op="linear", T=T, K=K, N=N, dtype=dtype, out=out, bias=bias, act=act, gated=gated,
                residual=residual, strided=strided)


def listed():
    return [
        # the two anchors of one asset at the 16 x 16 level of a 64 x 64 latent: latency counts
        _norm("norm_anchors_512", T=512, C=512),
        # all six views of 64 x 64 tokens on a full step, before the projection to queries, keys and values in 8 bits
        _norm("norm_full_step_24576", T=24576, C=2048),
        # foreground tokens of one asset, a residual stream kept in f32, 20 heads of 80
        _norm("norm_ragged_f32_residual", T=5391, C=1600, dtype="f16", residual="f32", out="f16"),
        # the attention's output of two anchors before its projection: 16 heads of 128
        _quantize("quantize_heads_8192", T=8192, C=2048),
        # foreground tokens' hidden rows of a feed-forward before its second product
        _quantize("quantize_hidden_ragged_f16", T=20001, C=8192, dtype="f16"),
        # scales, shifts and gates of a block from the time embedding, a row for each of four assets: the weights' bytes
        _linear("linear_time_rows_4", T=4, K=2048, N=12288),
        # two anchors at the 16 x 16 level, 8 heads of 64: the smallest projection of a cached step
        _linear("linear_anchors_512", T=512, K=512, N=1536, bias=False),
        # the last projection, from the tokens of all views to the latents' patches (x0 is kept in f32)
        _linear("linear_tokens_to_x0", T=24576, K=2048, N=64, out="f32"),
        # queries, keys and values of all six views on a full step
        _linear("linear_qkv_24576", T=24576, K=2048, N=6144, bias=False),
        # the gated feed-forward of one asset's foreground tokens
        _linear("linear_gated_ragged_f16", T=5391, K=1600, N=6400, dtype="f16", out="f16", act="gelu", gated=True),
        # the feed-forward of all six views in 8 bits: up ...
        _linear("linear_8bit_up_24576", T=24576, K=2048, N=8192, dtype="e4m3", act="gelu_tanh"),
        # ... and down into the residual, for the two anchors of a cached step
        _linear("linear_8bit_down_8192", T=8192, K=8192, N=2048, dtype="e4m3", residual=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["add_rms_norm", "quantize_rows", "linear", "linear", "linear"])
    strided = rng.random() < 0.3
    if op != "linear":
        C = rng.choice([_log(rng, 8, 16384), 8 * _log(rng, 2, 1024), rng.choice([320, 512, 640, 1280, 2048, 4096])])
        T = _log(rng, 1, min(49152, 100000000 // C))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op == "quantize_rows":
            return dict(op=op, T=T, C=C, dtype=dtype, strided=strided)
        return dict(op=op, T=T, C=C, dtype=dtype, residual=rng.choice(["", dtype, dtype, "f32"]),
                    out=rng.choice([dtype, "e4m3", "e4m3"]), strided=strided)
    dtype = rng.choice(["bf16", "bf16", "f16", "e4m3", "e4m3"])
    K = rng.choice([16 * _log(rng, 1, 640), rng.choice([320, 640, 1280, 2048, 4096, 8192])])
    N = rng.choice([_log(rng, 4, 12288), 8 * _log(rng, 1, 1536), rng.choice([640, 1280, 2048, 4096])])
    gated = rng.random() < 0.25
    T = _log(rng, 1, max(1, min(32768, int(4.0e11 / (K * N * (2 if gated else 1))))))
    half = dtype if dtype != "e4m3" else rng.choice(["bf16", "f16"])
    return dict(op=op, T=T, K=K, N=N, dtype=dtype, out=rng.choice([half, half, half, "f32"]), bias=rng.random() < 0.6,
                act=rng.choice(["gelu", "gelu_tanh", "silu"] + ([] if gated else ["", "", ""])), gated=gated,
                residual=rng.random() < 0.4, strided=strided)


def _size(dtype):
    return DTYPES[dtype].itemsize


def work(case):
    T = case["T"]
    if case["op"] == "linear":
        K, N, rows = case["K"], case["N"], case["N"] * (2 if case["gated"] else 1)
        e, o = _size(case["dtype"]), _size(case["out"])
        return {"bytes": (T + rows) * K * e + T * N * o * (2 if case["residual"] else 1) + (4 * rows if case["bias"] else 0)
                + (4 * (T + rows) if case["dtype"] == "e4m3" else 0),
                "flops": 2 * T * rows * K}
    n = T * case["C"]
    if case["op"] == "quantize_rows":
        return {"bytes": n * (_size(case["dtype"]) + 1) + 4 * T, "flops": 3 * n}
    r = 2 * _size(case["residual"]) if case["residual"] else 0  # read, and written with x added
    return {"bytes": n * (_size(case["dtype"]) + r + _size(case["out"])) + 4 * case["C"] + (4 * T if case["out"] == "e4m3" else 0),
            "flops": n * (5 if case["out"] != "e4m3" else 8)}


# ---------------------------------------------------------------- prepare --
def _rows(x, strided):
    """The rows as they lie in a program: alone, or as the first columns of a wider buffer."""
    if not strided:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + 64), device=DEV, dtype=torch.float32).to(x.dtype)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _plain_quantize(y):
    """(values, scales) of rows in 32 bits."""
    scale = (y.abs().amax(-1) / E4M3_MAX).clamp_(min=TINY)
    return (y / scale[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T = case["T"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)

    def empty(shape, dtype):
        return torch.empty(shape, device=DEV, dtype=DTYPES[dtype])

    if case["op"] != "linear":
        C = case["C"]
        # some channels of a denoiser's rows are much larger than the others
        channels = torch.exp(0.5 * randn(C))
        s = dict(op=case["op"], x=_rows((randn(T, C) * channels).to(DTYPES[case["dtype"]]), case["strided"]))
        if case["op"] == "quantize_rows":
            return dict(s, out=empty((T, C), "e4m3"), scale=empty((T,), "f32"))
        s.update(weight=1 + 0.1 * randn(C), residual=None, residual_out=None, eps=1e-6, out=empty((T, C), case["out"]),
                 scale=empty((T,), "f32") if case["out"] == "e4m3" else None)
        if case["residual"]:
            s["residual"] = (2 * randn(T, C) * channels).to(DTYPES[case["residual"]])
            s["residual_out"] = torch.empty_like(s["residual"])
        return s

    K, N = case["K"], case["N"]
    rows = N * (2 if case["gated"] else 1)
    x, w = randn(T, K), randn(rows, K) * K ** -0.5
    s = dict(op="linear", x_scale=None, weight_scale=None, act=case["act"] or None, gated=case["gated"],
             bias=0.1 * randn(rows) if case["bias"] else None,
             residual=randn(T, N).to(DTYPES[case["out"]]) if case["residual"] else None, out=empty((T, N), case["out"]))
    if case["dtype"] == "e4m3":
        x, s["x_scale"] = _plain_quantize(x)
        w, s["weight_scale"] = _plain_quantize(w)
    else:
        x, w = x.to(DTYPES[case["dtype"]]), w.to(DTYPES[case["dtype"]])
    return dict(s, x=_rows(x, case["strided"]), weight=w)


# -------------------------------------------------------------------- run --
def run(s):
    if own:
        from paper_2608_13255_gb300 import geocache as gc
        if s["op"] == "linear":
            return [gc.linear(s["x"], s["weight"], bias=s["bias"], activation=s["act"], gated=s["gated"],
                              residual=s["residual"], x_scale=s["x_scale"], weight_scale=s["weight_scale"], out=s["out"])]
        if s["op"] == "quantize_rows":
            return list(gc.quantize_rows(s["x"], out=s["out"], scale=s["scale"]))
        gc.add_rms_norm(s["x"], residual=s["residual"], weight=s["weight"], eps=s["eps"], out=s["out"], scale=s["scale"],
                        residual_out=s["residual_out"])
        return [s[k] for k in ("out", "scale", "residual_out") if s[k] is not None]
    if s["op"] == "linear":
        return [_plain_linear(s)]
    if s["op"] == "quantize_rows":
        return list(_plain_quantize(s["x"].float()))
    h, written = s["x"].float(), []
    if s["residual"] is not None:
        stored = (h + s["residual"].float()).to(s["residual"].dtype)  # what the stream keeps is what is normalised
        h, written = stored.float(), [stored]
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * s["weight"]
    return (list(_plain_quantize(y)) if s["scale"] is not None else [y.to(s["out"].dtype)]) + written


def _plain_act(x, kind):
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    if kind == "gelu":
        return 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))
    if kind == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh((2 / math.pi) ** 0.5 * (x + 0.044715 * x * x * x)))
    return x


def _plain_linear(s):
    y = torch.matmul(s["x"].float(), s["weight"].float().T)
    if s["x_scale"] is not None:
        y = y * s["x_scale"][:, None] * s["weight_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["gated"]:
        value, gate = y.chunk(2, -1)
        y = value * _plain_act(gate, s["act"])
    else:
        y = _plain_act(y, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["out"].dtype)


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if s["op"] != "linear":
        h = s["x"].to(f64)
        if s["op"] == "quantize_rows":
            y, more = h, []
        else:
            more = []
            if s["residual"] is not None:
                more = [h + s["residual"].to(f64)]
                h = more[0].to(s["residual"].dtype).to(f64)
            y = h * s["weight"].to(f64) / torch.sqrt(h.pow(2).sum(-1, keepdim=True) / h.shape[-1] + s["eps"])
            if s["scale"] is None:
                return [y] + more
        scale = torch.maximum(y.max(-1).values, -y.min(-1).values) / E4M3_MAX
        scale = torch.where(scale < TINY, torch.full_like(scale, TINY), scale)
        return [y / scale.unsqueeze(-1), scale] + more
    x, w = s["x"].to(f64), s["weight"].to(f64)
    if s["x_scale"] is not None:
        x, w = x * s["x_scale"].to(f64).unsqueeze(-1), w * s["weight_scale"].to(f64).unsqueeze(-1)
    out = torch.zeros(s["out"].shape, device=DEV, dtype=f64) if s["residual"] is None else s["residual"].to(f64)
    N = out.shape[1]
    part = [torch.addmm(torch.zeros((), device=DEV, dtype=f64) if s["bias"] is None else s["bias"][n:n + N].to(f64),
                        x, w[n:n + N].T) for n in range(0, w.shape[0], N)]
    z = part[-1]
    if s["act"] == "silu":
        z = z * torch.sigmoid(z)
    elif s["act"] == "gelu":
        z = z * torch.special.ndtr(z)
    elif s["act"] == "gelu_tanh":  # (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u))
        z = z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
    return [out + (z if len(part) == 1 else part[0] * z)]


if __name__ == "__main__":  # the cases and what each cannot do without
    for c in listed() + [draw(random.Random(i)) for i in range(12)]:
        w = work(c)
        print("%-28s %10.1f MB %10.1f GFLOP  %s" % (c.get("name", "(drawn)"), w["bytes"] / 1e6, w["flops"] / 1e9,
                                                    "" if "name" in c else c))
