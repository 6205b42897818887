"""A small transformer over the voxels of a batch of clouds, distilled from a teacher's top logits, then run voxel by voxel.

The rows of a sparse tensor, in the order in which the library numbers them, are the tokens; clouds lie one after another.  A sparse
convolution makes their features, one block of layer norm and windowed attention (a few first voxels of every cloud stay visible) mixes
them, and a head gives a category per voxel:

  x = conv(f);  h = x + Wo attend(Wqkv norm1(x));  logits = Whead norm2(h);  loss = distill(logits, teacher's best logits)

train() runs the step forward and backward through the library's own calls (the projections are plain matrix products) and applies SGD;
generate() then feeds the trained block one voxel at a time through sp_window_attn_step and compares with the packed form.

  python examples/voxel_tokens.py [--steps 30] [--points 2048]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2012_13846_amd import binding as sp  # noqa: E402
from paper_2012_13846_amd import spgen  # noqa: E402

CHANNELS, HEADS, KV_HEADS, DIM, CLASSES, TOP = 64, 4, 2, 32, 40, 5
WINDOW = dict(left=64, sinks=4)
QKV = HEADS + 2 * KV_HEADS


def make_params(g):
    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    c = CHANNELS
    return {"conv": normal(27, c, 16) / (27 * 16) ** 0.5, "qkv": normal(QKV * DIM, c) / c ** 0.5, "out": normal(c, HEADS * DIM) / c ** 0.5,
            "head": normal(CLASSES, c) / c ** 0.5, "gamma1": torch.ones(c, device="cuda"), "beta1": torch.zeros(c, device="cuda"),
            "gamma2": torch.ones(c, device="cuda"), "beta2": torch.zeros(c, device="cuda")}


def split_heads(w):
    w = w.view(-1, QKV, DIM)
    return w[:, :HEADS], w[:, HEADS:HEADS + KV_HEADS], w[:, HEADS + KV_HEADS:]


def forward(p, kmap, feats, starts):
    """Everything that the backward pass needs, by name."""
    b = {k: p[k].bfloat16() for k in ("conv", "qkv", "out", "head")}
    s = {"b": b, "x": sp.sp_conv_fwd(kmap, feats, b["conv"])}
    s["n1"], s["mean1"], s["rstd1"] = sp.sp_layer_norm_fwd(s["x"], p["gamma1"], p["beta1"])
    s["w"] = s["n1"] @ b["qkv"].t()
    s["o"], s["lse"] = sp.sp_window_attn_fwd(*split_heads(s["w"]), starts, starts, **WINDOW)
    s["h"] = s["x"] + s["o"].view(-1, HEADS * DIM) @ b["out"].t()
    s["n2"], s["mean2"], s["rstd2"] = sp.sp_layer_norm_fwd(s["h"], p["gamma2"], p["beta2"])
    s["logits"] = s["n2"] @ b["head"].t()
    return s


def backward(p, s, dlogits, kmap, feats, starts):
    b, g = s["b"], {}
    g["head"] = dlogits.t().float() @ s["n2"].float()
    dh, g["gamma2"], g["beta2"] = sp.sp_layer_norm_bwd(s["h"], dlogits @ b["head"], p["gamma2"], s["mean2"], s["rstd2"])
    g["out"] = dh.t().float() @ s["o"].view(-1, HEADS * DIM).float()
    do = (dh @ b["out"]).view(-1, HEADS, DIM)
    dw = torch.empty_like(s["w"])                              # the three gradients go into the fused projection's
    sp.sp_window_attn_bwd(*split_heads(s["w"]), s["o"], do, s["lse"], starts, starts, **WINDOW, out=split_heads(dw))
    g["qkv"] = dw.t().float() @ s["n1"].float()
    dx, g["gamma1"], g["beta1"] = sp.sp_layer_norm_bwd(s["x"], dw @ b["qkv"], p["gamma1"], s["mean1"], s["rstd1"])
    g["conv"] = sp.sp_conv_bwd_weight(kmap, feats, dx + dh)    # the residual's gradient joins
    return g


def train(steps: int, points: int, seed: int = 0, log=print):
    """Returns (parameters, losses, the last forward pass's state, starts)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    raw = torch.from_numpy(spgen.coords_config(1, points / 20000)).cuda()
    coords = sp.sp_coords_build(raw, 1)
    kmap, _ = sp.sp_kmap_build(coords, 3, 1, 1)
    batch = coords.coords()[:, 0].contiguous()                 # ascending: the input lists cloud after cloud
    clouds = int(batch[-1]) + 1
    starts = torch.searchsorted(batch, torch.arange(clouds + 1, dtype=torch.int32, device="cuda")).to(torch.int32)
    feats = torch.randn((coords.n, 16), device="cuda", generator=g).bfloat16()
    teacher = forward(make_params(g), kmap, feats, starts)["logits"].float() * 4
    top, index = teacher.topk(TOP, dim=1)
    top, index = top.contiguous(), index.to(torch.int32)
    p = make_params(g)
    losses = []
    for i in range(steps):
        s = forward(p, kmap, feats, starts)
        loss, dlogits = sp.sp_distill(s["logits"], top, index, temperature=2.0)
        grads = backward(p, s, dlogits, kmap, feats, starts)
        for k, v in grads.items():
            p[k] -= 0.5 * v
        losses.append(loss)
    losses = [float(v) for v in losses]
    log(f"{coords.n} voxels in {clouds} clouds: distillation loss {losses[0]:.4f} -> {losses[-1]:.4f} in {steps} steps")
    return p, losses, forward(p, kmap, feats, starts), starts


def generate(s, starts, log=print):
    """The attention of every cloud's voxels, one at a time and all clouds at once, through a ring that holds the window and the
    first voxels only.  Returns the largest difference from the packed form."""
    q, k, v = split_heads(s["w"])
    first = starts.tolist()
    lens = [b - a for a, b in zip(first, first[1:])]
    cap = WINDOW["sinks"] + WINDOW["left"] + 1
    caches = [torch.zeros((len(lens), cap, KV_HEADS, DIM), dtype=q.dtype, device="cuda") for _ in range(2)]
    begin, length = torch.tensor(first[:-1], device="cuda"), torch.tensor(lens, device="cuda")
    worst = torch.zeros((), device="cuda")
    for t in range(max(lens)):
        alive = length > t
        row = begin + torch.where(alive, t, 0)
        o = sp.sp_window_attn_step(q[row].contiguous(), k[row].contiguous(), v[row].contiguous(), *caches,
                                   torch.where(alive, t, -1).to(torch.int32), left=WINDOW["left"], sinks=WINDOW["sinks"])
        diff = (o.float() - s["o"][row].float()).abs().amax(dim=(1, 2))
        worst = torch.maximum(worst, torch.where(alive, diff, 0.0).max())
    log(f"{max(lens)} steps through a ring of {cap}: at most {float(worst):.4f} off the packed form (values up to {float(s['o'].abs().max()):.2f})")
    return float(worst)


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--steps", type=int, default=30)
    a.add_argument("--points", type=int, default=2048)
    a = a.parse_args()
    _, _, state, st = train(a.steps, a.points)
    generate(state, st)
