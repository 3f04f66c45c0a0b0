"""The residual stream in front of a layer: its calls together as a model makes them, forward, backward, captured, and with an int8 projection."""
import os
import sys

import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200.layer import Vsa2Layer, Vsa2ResidualNorm

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def off(got, want):
    return float((got.double() - want.double()).norm() / want.double().norm())


def make_layer(hidden, projection="fp8", seed=0, dim=64):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    p = vb.make_params(1, 2, 2, dim, (4, 8, 8), select_mode=vb.PER_QUERY, topk=2)
    layer = Vsa2Layer(p, hidden, (16, 24, 24), projection=projection)
    w = (randn(layer.width, hidden) * hidden ** -0.5).to(BF)
    layer.set_weights(w, (randn(hidden, 2) * hidden ** -0.5).to(BF), None, None)
    return layer, w, gen


@pytest.mark.parametrize("stream_type", [BF, F])
def test_stream_and_layer_together(stream_type):
    """The norm's own 8-bit form goes into the projection: what comes out is what the layer makes of it, and the gradients of branch, residual and weight are those of the
    formulas in 64 bits at the gradient that the layer returns for its hidden states."""
    layer, _, gen = make_layer(264)
    rows = layer.rows
    stream = Vsa2ResidualNorm(rows, 264, p=0.2, seed=77)
    weight = 1 + 0.1 * torch.randn(264, generator=gen, device="cuda")
    stream.set_weights(weight)
    branch = torch.randn(1, rows, 264, generator=gen, device="cuda").to(BF)
    residual = torch.randn(1, rows, 264, generator=gen, device="cuda").to(stream_type)
    h, x, x8 = stream.forward(branch, residual)
    factor = ref.factors(77, 1, rows, 264, 0.2)
    assert torch.equal(h.view(rows, -1), ref.stream(branch.view(rows, -1), residual.view(rows, -1), factor))
    want, _ = ref.normed(h.view(rows, -1), weight, 1e-6)
    assert ((x.view(rows, -1).double() - want).abs() <= (2.0 ** -8 + 2.0 ** -18) * want.abs()).all()
    o = layer.forward(x, x8)
    # (x8 is of the unrounded x: a layer that quantises the rounded one is off by the roundings of both, 4 significant bits on a few values)
    assert off(o, layer.forward(x)) <= 0.05
    o = layer.forward(x, x8)
    d_o, d_h = torch.randn(o.shape, generator=gen, device="cuda").to(BF), torch.randn(h.shape, generator=gen, device="cuda").to(stream_type)
    grads = layer.backward(d_o)
    got = stream.backward(grads["dx"], d_h)
    d, dw, size, size_w = ref.gradients(h.view(rows, -1), grads["dx"].view(rows, -1), d_h.view(rows, -1), weight, 1e-6)
    assert ((got["d_residual"].view(rows, -1).double() - d).abs() <= 2.0 ** -17 * size + torch.finfo(stream_type).eps / 2 * d.abs()).all()
    f = factor.cuda()
    assert ((got["d_branch"].view(rows, -1).double() - d * f).abs() <= (2.0 ** -17 * size + (2.0 ** -8 + 2.0 ** -23) * d.abs()) * f).all()
    assert ((got["d_weight"].double() - dw).abs() <= 2.0 ** -15 * size_w).all()
    assert got["d_residual"].dtype == stream_type and got["d_branch"].dtype == BF
    layer.check_status()


def test_without_dropout_one_gradient_serves_both():
    stream = Vsa2ResidualNorm(50, 128)
    branch, residual = torch.randn(50, 128, device="cuda").to(BF), torch.randn(50, 128, device="cuda").to(BF)
    stream.forward(branch, residual)
    got = stream.backward(torch.randn(50, 128, device="cuda").to(BF))
    assert got["d_branch"] is got["d_residual"]


def test_serving_in_whole_numbers():
    """One token at a time and all at once: the same bits, as every sum is exact; near the fp8 layer and the unquantised product."""
    layer, w, gen = make_layer(256, "int8")
    stream = Vsa2ResidualNorm(layer.rows, 256, p=0.5, projection="int8")
    branch, residual = (torch.randn(1, layer.rows, 256, generator=gen, device="cuda").to(BF) for _ in range(2))
    h, x, x8 = stream.forward(branch, residual, training=False)
    assert torch.equal(h, residual + branch) and isinstance(x8, vb.Int8)
    o = layer.forward(x, x8)
    fp8, _, _ = make_layer(256)
    assert off(o, fp8.forward(x)) <= 0.1      # (two forms of 8 bits, 4 % and 1.5 % off in each product)
    packed = torch.empty(layer.rows, layer.width, dtype=BF, device="cuda")
    vb.vsa2_int8_matmul(x8, layer.w, packed, layer.ws_matmul)
    exact = x.view(layer.rows, -1).double() @ w.double().T
    # the largest of 256 values is about 3 of them: steps of 3 / 127, uniform errors of 0.29 steps, in either operand
    assert off(packed, exact) <= 0.015
    for row in (0, 100, 255):
        one = Vsa2ResidualNorm(1, 256, projection="int8")
        _, _, token = one.forward(branch[:, row:row + 1].contiguous(), residual[:, row:row + 1].contiguous(), training=False)
        c = torch.empty(1, layer.width, dtype=BF, device="cuda")
        vb.vsa2_int8_matmul(token, layer.w, c, layer.ws_matmul)
        assert torch.equal(token.values[0], x8.values[row]) and torch.equal(c[0], packed[row])
    with pytest.raises(RuntimeError):
        layer.backward(o)


def test_a_captured_step_draws_anew_and_equals_the_eager_one():
    """Forward and backward of the stream as a graph: at each replay another offset, and the same results as calls made one by one with it.  Two graphs share a workspace."""
    rows, cols, p = 300, 520, 0.3
    gen = torch.Generator(device="cuda").manual_seed(4)
    branch, residual, dx = (torch.randn(rows, cols, generator=gen, device="cuda").to(BF) for _ in range(3))
    weight = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
    stream = Vsa2ResidualNorm(rows, cols, p=p, seed=5)
    stream.set_weights(weight)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        stream.forward(branch, residual)
        stream.backward(dx)
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                h, x, x8 = stream.forward(branch, residual)
                got = stream.backward(dx)
            graphs.append(g)
            outs.append((h, x, x8, got))
    torch.cuda.synchronize()
    stream.rng.copy_(torch.tensor([5, 40], device="cuda"))
    eager = Vsa2ResidualNorm(rows, cols, p=p, seed=5)
    eager.set_weights(weight)
    eager.rng[1] = 40
    for step in range(4):
        graphs[step % 2].replay()
        h, x, x8, got = outs[step % 2]
        eh, ex, ex8 = eager.forward(branch, residual)
        want = eager.backward(dx)
        assert torch.equal(h, eh) and torch.equal(x, ex) and torch.equal(x8.values.float(), ex8.values.float()) and torch.equal(x8.scales, ex8.scales)
        assert all(torch.equal(got[k], want[k]) for k in want)
        assert torch.equal(h, ref.stream(branch, residual, ref.factors(5, 41 + step, rows, cols, p)))


def test_calls_on_two_streams_at_once():
    """Each with buffers of its own, one behind the other on its stream, as on one alone."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    jobs = []
    for k in range(2):
        rows, cols, n = 3000 + 700 * k, 1536, 1000
        j = {"x": torch.randn(rows, cols, generator=gen, device="cuda").to(BF), "r": torch.randn(rows, cols, generator=gen, device="cuda").to(BF), "b": vb.Int8.empty(n, cols),
             "h": torch.empty(rows, cols, dtype=BF, device="cuda"), "q": vb.Int8.empty(rows, cols), "c": torch.empty(rows, n, dtype=BF, device="cuda"),
             "dw": torch.empty(cols, device="cuda"), "dr": torch.empty(rows, cols, dtype=BF, device="cuda"), "ws": vb.int8_matmul_workspace(rows, n, cols),
             "ws_norm": torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")}
        vb.vsa2_int8_quantize(torch.randn(n, cols, generator=gen, device="cuda"), j["b"])
        jobs.append(j)

    def run(j):
        vb.vsa2_residual_norm_fwd(j["x"], j["r"], h=j["h"], y_int8=j["q"])
        vb.vsa2_int8_matmul(j["q"], j["b"], j["c"], j["ws"])
        vb.vsa2_residual_norm_bwd(j["h"], j["x"], j["r"], d_residual=j["dr"], d_weight=j["dw"], workspace=j["ws_norm"])

    outputs = lambda: [[j[k].clone() for k in ("h", "c", "dr", "dw")] for j in jobs]
    for j in jobs:
        run(j)
    torch.cuda.synchronize()
    want = outputs()
    streams = [torch.cuda.Stream() for _ in jobs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for j, s in zip(jobs, streams):
            with torch.cuda.stream(s):
                run(j)
    torch.cuda.synchronize()
    for a, b in zip(outputs(), want):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_the_stream_refuses_other_shapes_and_changes():
    stream = Vsa2ResidualNorm(64, 128)
    x = torch.zeros(64, 128, dtype=BF, device="cuda")
    with pytest.raises(RuntimeError):
        stream.backward(x)
    for bad in (torch.zeros(63, 128, dtype=BF, device="cuda"), torch.zeros(128, 64, dtype=BF, device="cuda"), torch.zeros(128, 64, dtype=BF, device="cuda").T):
        with pytest.raises(ValueError):
            stream.forward(bad, x)
    with pytest.raises(ValueError):
        stream.forward(x.half(), x)
    with pytest.raises(ValueError):
        stream.set_weights(torch.ones(127, device="cuda"))
    with pytest.raises(ValueError):
        Vsa2ResidualNorm(64, 128, p=1.0)
    with pytest.raises(ValueError):
        Vsa2ResidualNorm(64, 128, projection="fp4")
    h, _, _ = stream.forward(x, x)
    h += 1
    with pytest.raises(RuntimeError):
        stream.backward(x)
    layer, _, _ = make_layer(128)
    hidden = torch.zeros(1, layer.rows, 128, dtype=BF, device="cuda")
    for wrong in (vb.Int8.empty(layer.rows, 128), vb.Fp8.empty(layer.rows, 129), vb.Fp8.empty(layer.rows - 1, 128)):
        with pytest.raises(ValueError):
            layer.forward(hidden, wrong)


def test_the_example_runs_with_the_stream():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_layer
    losses = train_layer.train(steps=3, grid=(4, 8, 8), heads=2, dim=64, hidden=256, topk=2, norm=True, dropout=0.1)
    assert len(losses) == 3 and all(v == v for v in losses)
