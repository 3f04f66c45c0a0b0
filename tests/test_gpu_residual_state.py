"""What the residual stream's norm keeps between forward and backward: the generator's state of its own forward, whatever the shared one has become."""
import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200.layer import Vsa2ResidualNorm

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
ROWS, COLS, P = 60, 264, 0.3


def made(seed=5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    branch, residual, dx = (torch.randn(ROWS, COLS, generator=gen, device="cuda") for _ in range(3))
    return Vsa2ResidualNorm(ROWS, COLS, p=P, seed=seed), branch, residual, dx


def check(stream, h, dx, offset):
    """Gradients through the mask of this offset.  (fp32 throughout: the norm's 2^-17 of the terms, a product with the mask's factor.)"""
    got = stream.backward(dx)
    factor = ref.factors(5, offset, ROWS, COLS, P).cuda()
    d, dw, size, size_w = ref.gradients(h, dx, None, None, 1e-6)
    assert ((got["d_branch"].double() == 0) == ((factor == 0) | (got["d_residual"] == 0))).all()
    assert ((got["d_branch"].double() - d * factor).abs() <= (2.0 ** -17 * size + 2.0 ** -23 * d.abs()) * factor).all()
    assert ((got["d_residual"].double() - d).abs() <= 2.0 ** -17 * size + 2.0 ** -24 * d.abs()).all()


def test_backward_after_the_generator_was_set_anew():
    stream, branch, residual, dx = made()
    h, _, _ = stream.forward(branch, residual)
    stream.rng.copy_(torch.tensor([9, 70], device="cuda"))
    check(stream, h, dx, 1)
    assert stream.rng.tolist() == [9, 70]
    h, _, _ = stream.forward(branch, residual)
    assert torch.equal(h, ref.stream(branch, residual, ref.factors(9, 71, ROWS, COLS, P)))


def test_backward_after_a_forward_that_was_refused():
    stream, branch, residual, dx = made()
    h, _, _ = stream.forward(branch, residual)
    for bad in (branch[:-1], branch.half(), branch.cpu()):
        with pytest.raises(ValueError):
            stream.forward(bad, residual)
    check(stream, h, dx, 1)


def test_backward_after_a_captured_step_was_replayed():
    """The captured step counts on the device, which nothing on the host sees."""
    stream, branch, residual, dx = made()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        stream.forward(branch, residual)
        stream.backward(dx)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            captured_h, _, _ = stream.forward(branch, residual)
            captured = stream.backward(dx)
    torch.cuda.synchronize()
    h, _, _ = stream.forward(branch, residual)      # the second that has run
    for _ in range(3):
        graph.replay()                              # .. up to the fifth
    check(stream, h, dx, 2)
    assert stream.rng.tolist() == [5, 5]
    factor = ref.factors(5, 5, ROWS, COLS, P)
    assert torch.equal(captured_h, ref.stream(branch, residual, factor))
    assert ((captured["d_branch"] == 0) == ((factor.cuda() == 0) | (captured["d_residual"] == 0))).all()


def test_a_forward_that_was_refused_has_not_counted():
    stream, branch, residual, _ = made()
    for bad in ((branch[:-1], residual), (branch.half(), residual), (branch, residual[:, :-1]), (branch.cpu(), residual), (branch, residual.double())):
        with pytest.raises(ValueError):
            stream.forward(*bad)
    assert stream.rng.tolist() == [5, 0]
    h, _, _ = stream.forward(branch, residual)
    assert torch.equal(h, ref.stream(branch, residual, ref.factors(5, 1, ROWS, COLS, P))) and stream.rng.tolist() == [5, 1]


def test_other_weights_are_refused_also_where_they_lie_in_the_old_ones_place():
    """The first weights are let go of between forward and backward, and another tensor comes to have their identity and their address."""
    stream, branch, residual, dx = made()
    weight = torch.full((COLS,), 2.0, device="cuda")
    name = id(weight)
    stream.set_weights(weight)
    stream.forward(branch, residual)
    stream.set_weights(None)
    del weight
    others = []
    for _ in range(1000):
        others.append(torch.full((COLS,), 3.0, device="cuda"))
        if id(others[-1]) == name:
            break
    for other in (others[-1], None, others[0]):
        stream.set_weights(other)
        with pytest.raises(RuntimeError, match="changed between"):
            stream.backward(dx)


@pytest.mark.parametrize("branch_type,p", [(F, 0.0), (F, P), (BF, 0.0), (BF, P)])
def test_each_gradient_has_its_input_s_shape(branch_type, p):
    """Rows as they lie; a branch [tokens, hidden] beside a stream [batch, tokens, hidden], and the other way round."""
    _, branch, residual, dx = made()
    stream = Vsa2ResidualNorm(ROWS, COLS, p=p, seed=5)
    h, _, _ = stream.forward(branch.to(branch_type), residual)
    want = stream.backward(dx)
    for of_branch, of_residual in (((ROWS, COLS), (2, ROWS // 2, COLS)), ((1, ROWS, COLS), (ROWS, COLS)), ((ROWS, 1, COLS), (3, 4, 5, COLS))):
        other = Vsa2ResidualNorm(ROWS, COLS, p=p, seed=5)
        assert torch.equal(other.forward(branch.to(branch_type).view(of_branch), residual.view(of_residual))[0], h.view(of_residual))
        got = other.backward(dx)
        assert got["d_branch"].shape == of_branch and got["d_residual"].shape == of_residual
        assert got["d_branch"].dtype == branch_type and torch.equal(got["d_branch"].view(ROWS, COLS), want["d_branch"])
        assert torch.equal(got["d_residual"].view(ROWS, COLS), want["d_residual"])


@pytest.mark.parametrize("projection", ["fp8", "int8"])
def test_no_rows(projection):
    stream = Vsa2ResidualNorm(0, COLS, p=P, projection=projection)
    branch, residual = torch.empty(2, 0, COLS, dtype=BF, device="cuda"), torch.empty(0, COLS, device="cuda")
    h, x, x8 = stream.forward(branch, residual)
    assert h.shape == x.shape == x8.shape == (0, COLS) and (h.dtype, x.dtype) == (F, BF)
    got = stream.backward(torch.empty(0, COLS, device="cuda"), torch.empty(0, COLS, device="cuda"))
    assert got["d_branch"].shape == (2, 0, COLS) and got["d_residual"].shape == (0, COLS)
    assert got["d_weight"].shape == (COLS,) and not got["d_weight"].any()
