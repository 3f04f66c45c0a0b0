"""The gate's share of the layer: output and all gradients against the layer with its gated coarse branch in 64 bits.

Bounds as for the layer without a gate (outputs 1 %; gradients that pass the 8-bit products 6 %).  dW_g and the norm weights' gradients pass none: the gate's dz is rounded to bf16 (2^-9 at
most), and what it is made of is the attention's output, 1 % off at most."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200.layer import Vsa2Layer

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def cubes_of(grid, device):
    """Cube of every token of the raster, and the cubes' number of tokens."""
    r = torch.arange(grid[0] * grid[1] * grid[2], device=device)
    t, h, w = r // (grid[1] * grid[2]), r // grid[2] % grid[1], r % grid[2]
    n = [-(-g // 4) for g in grid]
    cube = (t // 4 * n[1] + h // 4) * n[2] + w // 4
    return cube, torch.bincount(cube, minlength=n[0] * n[1] * n[2]).double()


def reference(p, grid, channels, hidden_states, raw, w, w_g, qw, kw):
    """The layer in 64 bits: `hidden_states` as the projection takes them (leaf), `raw` as the gate does (leaf)."""
    batch, n, _ = raw.shape
    hq, hk, dim = p.heads_q, p.heads_kv, p.head_dim
    video = grid[0] * grid[1] * grid[2]
    heads = (hidden_states @ w.T).view(batch, n, hq + 2 * hk, dim).transpose(1, 2)
    r = torch.arange(n, device=raw.device)
    pos = (torch.stack([r // (grid[1] * grid[2]), r // grid[2] % grid[1], r % grid[2]], -1) * (r < video).unsqueeze(-1)).double()
    angle = torch.cat([pos[:, i:i + 1] * torch.tensor([1e4 ** (-2.0 * j / c) for j in range(c // 2)], dtype=torch.float64, device=raw.device)
                       for i, c in enumerate(channels)], -1)

    def turn(v):
        z = torch.view_as_complex(v[..., :2 * angle.shape[1]].unflatten(-1, (-1, 2)).contiguous()) * torch.polar(torch.ones_like(angle), angle)
        return torch.cat([torch.view_as_real(z).flatten(-2), v[..., 2 * angle.shape[1]:]], -1)

    norm = lambda v, g: v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-6) * g
    q, k, v = turn(norm(heads[:, :hq], qw)), turn(norm(heads[:, hq:hq + hk], kw)), heads[:, hq + hk:]
    k, v = k.repeat_interleave(hq // hk, 1), v.repeat_interleave(hq // hk, 1)
    fine = torch.softmax(q @ k.transpose(-1, -2) * dim ** -0.5, -1) @ v
    cube, count = cubes_of(grid, raw.device)
    pool = lambda t: torch.zeros(*t.shape[:2], len(count), dim, dtype=torch.float64, device=raw.device).index_add(2, cube, t[:, :, :video]) / count.unsqueeze(-1)
    coarse = torch.softmax(pool(q) @ pool(k).transpose(-1, -2) * dim ** -0.5, -1) @ pool(v)
    gate = torch.tanh(raw[:, :video] @ w_g).transpose(1, 2)
    return torch.cat([fine[:, :, :video] + gate.unsqueeze(-1) * coarse[:, :, cube], fine[:, :, video:]], 2)


def problem(batch, hq, hk, dim, grid, text, hidden, gate_size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(hidden + hq)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    channels = (16, 24, 24) if dim == 64 else (44, 42, 42)
    p = vb.make_params(batch, hq, hk, dim, grid, select_mode=vb.PER_QUERY, topk=1 << 20, text_len=text)
    layer = Vsa2Layer(p, hidden, channels)
    # a share that all tokens have in common, so that the cubes' means (and with them the coarse branch and its gate's gradient) are of the size of a token's values
    x = (randn(batch, layer.tokens, hidden) + randn(batch, 1, hidden)).to(BF)
    w, w_g = (randn(layer.width, hidden) * hidden ** -0.5).to(BF), (randn(hidden, hq) * gate_size * hidden ** -0.5).to(BF)
    qw, kw = 1 + 0.1 * randn(dim), 1 + 0.1 * randn(dim)
    layer.set_weights(w, w_g, qw, kw)
    return layer, channels, x, w_g, qw, kw, randn(batch, hq, layer.tokens, dim).to(BF)


@pytest.mark.parametrize("batch,hq,hk,dim,grid,text,hidden", [(1, 4, 2, 64, (4, 8, 8), 0, 256), (2, 3, 3, 128, (3, 5, 9), 21, 328), (3, 6, 2, 64, (5, 6, 7), 0, 136)])
def test_layer_with_a_gate_against_autograd(batch, hq, hk, dim, grid, text, hidden):
    layer, channels, x, w_g, qw, kw, d_o = problem(batch, hq, hk, dim, grid, text, hidden)
    o = layer.forward(x)
    got = layer.backward(d_o)
    layer.check_status()
    a = vb.Fp8.empty(layer.rows, hidden)
    vb.vsa2_fp8_quantize(x.view(-1, hidden), a)
    leaf = lambda t: t.double().requires_grad_()
    X, raw, W, WG, QW, KW = (leaf(t) for t in (a.dequantize().view(x.shape), x, layer.w.dequantize(), w_g, qw, kw))
    O = reference(layer.p, grid, channels, X, raw, W, WG, QW, KW)
    O.backward(d_o.double())
    dx = X.grad + raw.grad
    assert float(raw.grad.norm()) >= 0.2 * float(dx.norm())          # (the gate's part is well above the bound)
    assert off(o, O.detach()) <= 0.01
    assert off(got["dx"], dx) <= 0.06
    assert off(got["dw_qkv"], W.grad) <= 0.06
    assert off(got["dw_g"], WG.grad) <= 0.02
    assert off(got["dq_weight"], QW.grad) <= 0.02 and off(got["dk_weight"], KW.grad) <= 0.02
