#!/usr/bin/env python
"""Trains one attention layer on a clip, from hidden states to the attention's output and back, through the library's calls alone (paper_2609_32882_b200/layer.py).

    python examples/train_layer.py [--steps 20] [--grid 8,16,16] [--heads 12] [--hidden 1536] [--text 0] [--norm] [--dropout 0.1]

A layer with random weights learns the output of another one; plain gradient descent on fp32 master weights.  Prints the loss of every step.
With --norm its hidden states are the norm of a residual stream and a branch, of which --dropout drops a share in each step; the norm's weights learn too.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_32882_b200 import binding as vb  # noqa: E402
from paper_2609_32882_b200.layer import Vsa2Layer, Vsa2ResidualNorm  # noqa: E402


def master_weights(gen, width, hidden, heads, dim):
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return {"w_qkv": randn(width, hidden) * hidden ** -0.5, "w_g": randn(hidden, heads) * 0.5 * hidden ** -0.5,
            "q_weight": 1 + 0.1 * randn(dim), "k_weight": 1 + 0.1 * randn(dim)}


def put(layer, w):
    layer.set_weights(w["w_qkv"].bfloat16(), w["w_g"].bfloat16(), w["q_weight"], w["k_weight"])


def train(steps=20, grid=(8, 16, 16), heads=12, dim=128, hidden=1536, text=0, topk=8, rate=0.5, seed=0, norm=False, dropout=0.0):
    """Losses of the steps, largest first if all goes well."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    p = vb.make_params(1, heads, heads, dim, grid, select_mode=vb.PER_QUERY, topk=topk, text_len=text)
    layer = Vsa2Layer(p, hidden, (dim - 2 * (dim // 6 * 2), dim // 6 * 2, dim // 6 * 2))
    x = torch.randn(1, layer.tokens, hidden, generator=gen, device="cuda").bfloat16()
    put(layer, master_weights(gen, layer.width, hidden, heads, dim))
    names = [("w_qkv", "dw_qkv"), ("w_g", "dw_g"), ("q_weight", "dq_weight"), ("k_weight", "dk_weight")]
    stream = None
    if norm:
        stream = Vsa2ResidualNorm(layer.rows, hidden, p=dropout, seed=seed)
        residual = torch.randn(x.shape, generator=gen, device="cuda")
        stream.set_weights(1 + 0.1 * torch.randn(hidden, generator=gen, device="cuda"))
        names.append(("norm", "d_norm"))

    def forward(training):
        if stream is None:
            return layer.forward(x)
        _, y, y8 = stream.forward(x, residual, training)
        return layer.forward(y, y8)

    target = forward(False).float()
    w = master_weights(gen, layer.width, hidden, heads, dim)
    if norm:
        w["norm"] = torch.ones(hidden, device="cuda")
    losses = []
    for _ in range(steps):
        put(layer, w)
        if norm:
            stream.set_weights(w["norm"])
        diff = forward(True).float() - target
        losses.append(float(diff.square().mean() / target.square().mean()))
        grads = layer.backward((diff / target.norm()).bfloat16())
        if norm:
            grads["d_norm"] = stream.backward(grads["dx"])["d_weight"]
        for name, g in names:
            w[name] -= rate * grads[g] * w[name].norm() / grads[g].norm().clamp(min=1e-30) / 10
    layer.check_status()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--grid", default="8,16,16")
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--hidden", type=int, default=1536)
    ap.add_argument("--text", type=int, default=0)
    ap.add_argument("--norm", action="store_true")
    ap.add_argument("--dropout", type=float, default=0.0)
    a = ap.parse_args()
    if a.dropout and not a.norm:
        ap.error("--dropout is that of the residual stream's branch: with --norm")
    for i, loss in enumerate(train(a.steps, tuple(int(v) for v in a.grid.split(",")), a.heads, hidden=a.hidden, text=a.text, norm=a.norm, dropout=a.dropout)):
        print(f"step {i}: loss {loss:.5f}")
