"""A sampler loop whose denoiser is one multi-view attention block, on seeded synthetic geometry.

Full steps run the block on all views; cached steps run it on the anchors alone (Sec. 3.2, batch-sliced anchor forward):
their rows are packed, keep the rotary slots of the N-view layout, and attend to each other inside their asset; the
library transports their change to the other views.  Background tokens take no part, so each asset is a packed sequence
of its own length.  The projections are torch products; the norms with the rotation, the attention, the packing, the
transport and the reconstruction are the library's.

    python examples/anchor_attention.py [--workload hunyuan64] [--assets 2] [--heads 8] [--dim 64] [--steps 10]
"""
import argparse
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2608_13255_gb300 import geocache as gc  # noqa: E402
from paper_2608_13255_gb300 import synth  # noqa: E402


def rotary_table(N, H, W, D):
    """Rotation over three axes (view, row, column) for the slots (v * H + y) * W + x: a range of pairs for each."""
    slot = torch.arange(N * H * W, dtype=torch.int32, device="cuda")
    table = torch.empty((N * H * W, D // 2, 2), device="cuda")
    per = D // 2 // 3
    first = 0
    for pos, pairs in ((slot // (H * W), D // 2 - 2 * per), (slot // W % H, per), (slot % W, per)):
        gc.rope_table(rot=2 * pairs, theta=100.0, pos=pos.contiguous(), table=table, first_pair=first)
        first += pairs
    return table


class Block:
    """x0 of the views that are given: latents -> heads -> attention inside each asset -> latents."""

    def __init__(self, w, heads, kv_heads, D, seed=0):
        self.w, self.Hq, self.Hk, self.D = w, heads, kv_heads, D
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.into = (r(w.C + 3, (heads + 2 * kv_heads) * D) / (w.C + 3) ** 0.5).to(torch.bfloat16)
        self.back = (r(heads * D, w.C) / (heads * D) ** 0.5).to(torch.bfloat16)
        self.q_weight, self.k_weight = 1 + 0.1 * r(D), 1 + 0.1 * r(D)
        self.table = rotary_table(w.N, w.H, w.W, D)
        self.pos = torch.from_numpy(w.pos).cuda()
        self.valid = torch.from_numpy(w.valid).cuda()
        self.kept = {}  # token lists and plans of the view sets that the rotation comes back to

    def rows(self, views):
        """Foreground tokens of the views: their places among the packed rows, their slots, and the attention's plan."""
        if views not in self.kept:
            w = self.w
            fg = self.valid[:, list(views)].reshape(w.B, -1) != 0
            place = fg.flatten().nonzero().squeeze(1)
            token = place % (len(views) * w.H * w.W)
            first = torch.tensor(views, device="cuda") * (w.H * w.W)
            slots = (first[token // (w.H * w.W)] + token % (w.H * w.W)).to(torch.int32)
            lens = fg.sum(1).tolist()
            self.kept[views] = (place, slots, gc.attention_plan(lens, lens, self.Hq, self.Hk, self.D))
        return self.kept[views]

    def qkv(self, x, views):
        w = self.w
        place, slots, plan = self.rows(views)
        n = len(views)
        latents = x.float().permute(0, 1, 3, 4, 2).reshape(w.B * n * w.H * w.W, w.C)
        pos = self.pos
        if n < w.N:  # the anchors' rows of a structural input
            packed = torch.empty((w.B, n) + tuple(pos.shape[2:]), device="cuda")
            gc.pack_anchors(pos, packed, views)
            pos = packed
        features = torch.cat([latents, pos.reshape(-1, 3)], 1)[place].to(torch.bfloat16)
        qkv = (features @ self.into).view(-1, self.Hq + 2 * self.Hk, self.D)
        return qkv, place, slots, plan

    def __call__(self, x, views):
        views = tuple(views)
        w, Hq, Hk = self.w, self.Hq, self.Hk
        qkv, place, slots, plan = self.qkv(x, views)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        gc.qk_norm_rope(q, k, self.table, slots, self.q_weight, self.k_weight, q_out=q, k_out=k)  # in place
        out = gc.attention(plan, q, k, v)
        x0 = torch.zeros((w.B * len(views) * w.H * w.W, w.C), device="cuda")
        x0[place] = (out.reshape(len(place), -1) @ self.back).float()
        return x0.view(w.B, len(views), w.H, w.W, w.C).permute(0, 1, 4, 2, 3).contiguous()


def run(block, steps, every=5, a=2, seed=0):
    """The loop; returns (x at the end, the x0 cache)."""
    w = block.w
    corr = gc.build_sparse_corr(block.pos, block.valid, torch.from_numpy(w.cams).cuda(), K=4)
    ws = torch.empty(max(1, corr.workspace_floats(w.C)), device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((w.B, w.N, w.C, w.H, w.W), generator=g, device="cuda").to(torch.bfloat16)
    x_next, x0 = torch.empty_like(x), torch.zeros(x.shape, device="cuda")
    anchor_rows = torch.empty((w.B, a) + tuple(x.shape[2:]), device="cuda", dtype=x.dtype)
    for t in range(steps):
        s, s_next = 1.0 - t / steps, 1.0 - (t + 1) / steps
        recon = gc.make_recon("fm_euler", sigma=s, sigma_next=s_next)
        anchors, full = gc.rotate_anchors(w.N, a, t, steps, {"kind": "every_k", "k": every})
        if full:
            x0 = block(x, range(w.N))
            gc.reconstruct(x, x0, x_next, recon)
        else:
            gc.pack_anchors(x, anchor_rows, anchors)
            gc.transport_step(corr, anchors, w.C, block(anchor_rows, anchors), x0, x0, x, x_next, recon, workspace=ws)
        x, x_next = x_next, x
    return x, x0


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="hunyuan64")
    ap.add_argument("--assets", type=int, default=2)
    ap.add_argument("--heads", type=int, default=8)
    ap.add_argument("--kv-heads", type=int, default=0, help="default: --heads")
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--steps", type=int, default=10)
    o = ap.parse_args()
    w = synth.make_workload(o.workload, B=o.assets)
    block = Block(w, o.heads, o.kv_heads or o.heads, o.dim)
    run(block, o.steps)
    gc.device_status()
    torch.cuda.synchronize()
    t = time.perf_counter()
    x, x0 = run(block, o.steps)
    torch.cuda.synchronize()
    gc.device_status()
    print("%s: %d assets x %d views, %d steps: %.2f ms; x0 rms %.4f" %
          (o.workload, w.B, w.N, o.steps, 1e3 * (time.perf_counter() - t), float(x0.square().mean().sqrt())))


if __name__ == "__main__":
    main()
