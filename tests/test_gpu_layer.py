"""The calls between hidden states and attention together, as a layer makes them: outputs and gradients against the layer's definition in 64 bits.

With every block kept and the gate's weights zero the attention is dense softmax attention and has no coarse part in its output, so torch's autograd in 64 bits gives the whole layer.
Bounds (derived): values are rounded to 4 significant bits, 2^-5 to 2^-4 of themselves at most, 2.7 % on average over a binade; a product of two such
matrices is 3.8 % off in its norm, and what comes behind it keeps that share (the reference holds the layer's own rounded x and W, so its forward's projection has only bf16's rounding, 0.3 %
with the attention's; gradients are rounded in the layer alone)."""
import os
import sys

import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200.layer import Vsa2Layer

pytestmark = pytest.mark.gpu


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("batch,hq,hk,dim,grid,text,hidden", [(1, 4, 2, 64, (4, 8, 8), 0, 256), (2, 3, 3, 128, (3, 5, 9), 21, 328)])
def test_layer_against_autograd(batch, hq, hk, dim, grid, text, hidden):
    gen = torch.Generator(device="cuda").manual_seed(hidden)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    channels = (16, 24, 24) if dim == 64 else (44, 42, 42)
    p = vb.make_params(batch, hq, hk, dim, grid, select_mode=vb.PER_QUERY, topk=1 << 20, text_len=text)
    layer = Vsa2Layer(p, hidden, channels)
    n = layer.tokens
    x = randn(batch, n, hidden).bfloat16()
    w, qw, kw = (randn(layer.width, hidden) * hidden ** -0.5).bfloat16(), 1 + 0.1 * randn(dim), 1 + 0.1 * randn(dim)
    layer.set_weights(w, torch.zeros(hidden, hq, dtype=torch.bfloat16, device="cuda"), qw, kw)
    o = layer.forward(x)
    d_o = randn(*o.shape).bfloat16()
    got = layer.backward(d_o)
    layer.check_status()

    a = vb.Fp8.empty(batch * n, hidden)
    vb.vsa2_fp8_quantize(x.view(-1, hidden), a)
    X = a.dequantize().double().view(batch, n, hidden).requires_grad_()
    W = layer.w.dequantize().double().requires_grad_()
    QW, KW = qw.double().requires_grad_(), kw.double().requires_grad_()
    heads = (X @ W.T).view(batch, n, hq + 2 * hk, dim).transpose(1, 2)
    t, h, wd = grid
    r = torch.arange(n, device="cuda")
    pos = (torch.stack([r // (h * wd), r // wd % h, r % wd], -1) * (r < t * h * wd).unsqueeze(-1)).double()
    angle = torch.cat([pos[:, i:i + 1] * torch.tensor([1e4 ** (-2.0 * j / c) for j in range(c // 2)], dtype=torch.float64, device="cuda")
                       for i, c in enumerate(channels)], -1)

    def turn(v):
        z = torch.view_as_complex(v[..., :2 * angle.shape[1]].unflatten(-1, (-1, 2)).contiguous()) * torch.polar(torch.ones_like(angle), angle)
        return torch.cat([torch.view_as_real(z).flatten(-2), v[..., 2 * angle.shape[1]:]], -1)

    norm = lambda v, g: v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-6) * g
    q, k, v = turn(norm(heads[:, :hq], QW)), turn(norm(heads[:, hq:hq + hk], KW)), heads[:, hq + hk:]
    k, v = k.repeat_interleave(hq // hk, 1), v.repeat_interleave(hq // hk, 1)
    O = torch.softmax(q @ k.transpose(-1, -2) * dim ** -0.5, -1) @ v
    O.backward(d_o.double())
    assert off(o, O.detach()) <= 0.01
    assert off(got["dx"], X.grad) <= 0.06
    assert off(got["dw_qkv"], W.grad) <= 0.06
    assert off(got["dq_weight"], QW.grad) <= 0.02 and off(got["dk_weight"], KW.grad) <= 0.02


def test_the_example_learns():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_layer
    losses = train_layer.train(steps=12, grid=(4, 8, 8), heads=2, dim=64, hidden=256, topk=2)
    assert losses[-1] < 0.8 * losses[0] and min(losses) == min(losses[-4:])
    with_text = train_layer.train(steps=3, grid=(3, 5, 7), heads=2, dim=64, hidden=264, text=19, topk=2)
    assert all(v == v for v in with_text)


def test_layer_refuses_other_shapes():
    p = vb.make_params(1, 2, 2, 64, (4, 8, 8), select_mode=vb.PER_QUERY, topk=2)
    layer = Vsa2Layer(p, 128, (16, 24, 24))
    with pytest.raises(ValueError):
        layer.forward(torch.zeros(1, 255, 128, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        Vsa2Layer(vb.make_params(1, 2, 2, 64, (4, 8, 8), topk=2, out_dtype=vb.F32), 128, (16, 24, 24))
