"""The gate's share of the layer: output and all gradients against the layer with its gated coarse branch in 64 bits, and how the two parts of dX come together.

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


@pytest.mark.parametrize("batch,grid,text", [(1, (4, 8, 8), 0), (2, (3, 5, 9), 21)])
def test_parts_of_dx(batch, grid, text, monkeypatch):
    """dX = the product's result + sum_h dz_h w_g, and in text rows the product's alone.  With the layer's own product and dz (as it rounds them, to bf16) the sum is known to
    2^-20, and one rounding to bf16 is left: its squares average a twelfth of the unit's."""
    hidden = 256
    layer, _, x, w_g, _, _, d_o = problem(batch, 4, 2, 64, grid, text, hidden, 4.0)
    video = grid[0] * grid[1] * grid[2]
    products, dgates = [], []
    matmul, attn_backward = vb.vsa2_fp8_matmul, layer.attn.backward

    def recorded(a, b, c, *rest, **kw):
        matmul(a, b, c, *rest, **kw)
        products.append(c.clone())

    def recorded_backward(*a, **kw):
        out = attn_backward(*a, **kw)
        dgates.append(out[3].clone())
        return out

    layer.forward(x)
    gate = layer.saved[6].clone()
    monkeypatch.setattr(vb, "vsa2_fp8_matmul", recorded)
    monkeypatch.setattr(layer.attn, "backward", recorded_backward)
    dx = layer.backward(d_o)["dx"]
    product = next(c for c in products if c.shape == (layer.rows, hidden) and c.dtype == BF).view(dx.shape)
    dz = (dgates[0] * (1 - gate * gate)).to(BF).double()
    gates_part = dz.transpose(1, 2) @ w_g.double().T
    want = product.double()
    assert torch.equal(dx[:, video:], product[:, video:])
    want[:, :video] += gates_part
    unit = torch.ldexp(torch.ones_like(want), torch.frexp(want)[1] - 8)[:, :video]
    assert float(gates_part.norm()) >= 2 * float(product[:, :video].norm())      # (whose own rounding would show)
    err = (dx.double() - want)[:, :video]
    assert float((err ** 2).sum()) <= 1.2 * float((unit ** 2).sum()) / 12


@pytest.mark.parametrize("out_dtype", [vb.BF16, vb.F32])
@pytest.mark.parametrize("batch,heads,grid,hidden,rows", [(1, 5, (3, 5, 7), 72, 105), (2, 40, (4, 8, 16), 264, 600), (3, 64, (2, 9, 11), 136, 198), (2, 17, (1, 1, 3), 8, 4)])
def test_gate_backward_onto_a_gradient(batch, heads, grid, hidden, rows, out_dtype):
    """vsa2_gate_bwd_add against vsa2_gate_bwd in fp32: the same products, added to what is there and rounded once; rows behind the video's and dW_g as they are without."""
    gen = torch.Generator(device="cuda").manual_seed(heads)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    n = grid[0] * grid[1] * grid[2]
    make = lambda dtype: vb.make_params(batch, heads, heads, 64, grid, topk=1, out_dtype=dtype)
    p = make(out_dtype)
    x, w, gate, dgate = randn(batch, n, hidden).to(BF), randn(hidden, heads).to(BF), torch.tanh(randn(batch, heads, n)), randn(batch, heads, n)
    ws = torch.empty(vb.vsa2_gate_bwd_workspace_bytes(p, hidden), dtype=torch.uint8, device="cuda")
    dw, part = [torch.empty(hidden, heads, device="cuda") for _ in range(2)], torch.empty(batch, n, hidden, device="cuda")
    vb.vsa2_gate_bwd(make(vb.F32), hidden, x, w, gate, dgate, dw[0], part, ws)
    before = randn(batch, rows, hidden).to(torch.float32 if out_dtype == vb.F32 else BF)
    dx = before.clone()
    vb.vsa2_gate_bwd_add(p, hidden, x, w, gate, dgate, dw[1], dx, ws)
    want = before.clone()
    want[:, :n] = (before[:, :n].float() + part).to(before.dtype)
    assert torch.equal(dx, want) and torch.equal(dw[0], dw[1])
    for bad in (dx.half(), dx[:, :n - 1], dx[..., :-1], dx.transpose(1, 2), dx[:1, :, :].expand(batch + 1, rows, hidden)):
        with pytest.raises(ValueError):
            vb.vsa2_gate_bwd_add(p, hidden, x, w, gate, dgate, dw[1], bad, ws)
