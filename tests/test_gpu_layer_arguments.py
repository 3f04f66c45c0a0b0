"""What the layer refuses: it hands plain addresses to the attention and to the gate, which take their sizes and types from the layer's parameters."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200.layer import Vsa2Layer

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def problem(batch=1, text=0, hidden=128):
    p = vb.make_params(batch, 4, 2, 64, (2, 4, 8), select_mode=vb.PER_QUERY, topk=2, text_len=text)
    layer = Vsa2Layer(p, hidden, (16, 24, 24))
    gen = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    weights = [(randn(layer.width, hidden) * hidden ** -0.5).to(BF), (randn(hidden, 4) * hidden ** -0.5).to(BF), 1 + 0.1 * randn(64), 1 + 0.1 * randn(64)]
    return layer, weights, randn(batch, layer.tokens, hidden).to(BF), randn(batch, 4, layer.tokens, 64).to(BF)


@pytest.mark.parametrize("i,change", [
    (0, lambda w: w[:-1]), (0, lambda w: w.T.contiguous()), (0, lambda w: w.half()),
    (1, lambda w: w.float()), (1, lambda w: w[:, :3].contiguous()), (1, lambda w: w[:-8]), (1, lambda w: w.T), (1, lambda w: w.half()), (1, lambda w: w.cpu()),
    (2, lambda w: w.to(BF)), (2, lambda w: w[:63]), (3, lambda w: torch.cat([w, w])),
])
def test_weights_that_do_not_fit(i, change):
    layer, w, x, _ = problem()
    layer.set_weights(*w)
    want = layer.forward(x)
    bad = list(w)
    bad[i] = change(w[i])
    with pytest.raises(ValueError):
        layer.set_weights(*bad)
    assert torch.equal(layer.forward(x), want)            # (nothing of it was taken)


@pytest.mark.parametrize("change", [lambda t: t.float(), lambda t: t.half(), lambda t: t[:, :-1], lambda t: t.cpu(), lambda t: t.transpose(-1, -2).contiguous().transpose(-1, -2)])
def test_hidden_states_and_gradients_that_do_not_fit(change):
    layer, w, x, d_o = problem()
    layer.set_weights(*w)
    with pytest.raises(ValueError):
        layer.forward(change(x))
    layer.forward(x)
    with pytest.raises(ValueError):
        layer.backward(change(d_o))
    layer.backward(d_o)
    layer.check_status()


def test_master_weights_in_fp32_and_norms_without_weights():
    layer, w, x, _ = problem()
    layer.set_weights(w[0].float(), w[1], torch.ones(64, device="cuda"), torch.ones(64, device="cuda"))
    want = layer.forward(x)
    room = torch.zeros(layer.width, 200, dtype=BF, device="cuda")
    room[:, 3:131] = w[0]
    layer.set_weights(room[:, 3:131], w[1], None, None)            # (rows of a larger matrix)
    assert torch.equal(layer.forward(x), want)


@pytest.mark.parametrize("change", ["x", "o", "w_g", "q_weight", "k_weight", "set_weights"])
def test_backward_of_a_forward_whose_tensors_have_changed(change):
    """Gradients would be of a mixture of two states: x is quantised again for dW, the weights are read again."""
    layer, w, x, d_o = problem()
    layer.set_weights(*w)
    o = layer.forward(x)
    want = layer.backward(d_o)
    if change == "set_weights":
        layer.set_weights(*w)
    else:
        {"x": x, "o": o, "w_g": w[1], "q_weight": w[2], "k_weight": w[3]}[change].mul_(1)
    with pytest.raises(RuntimeError, match=change):
        layer.backward(d_o)
    layer.forward(x)
    again = layer.backward(d_o)
    assert all(torch.equal(want[k], again[k]) for k in want)


def test_calls_before_those_they_need():
    layer, w, x, d_o = problem()
    with pytest.raises(RuntimeError, match="set_weights"):
        layer.forward(x)
    layer.set_weights(*w)
    with pytest.raises(RuntimeError, match="forward"):
        layer.backward(d_o)


def test_tensors_of_inference_mode():
    with torch.inference_mode():
        layer, w, x, d_o = problem()
        layer.set_weights(*w)
        layer.forward(x)
        layer.backward(d_o)
