"""A layer that only serves holds nothing between calls that only a backward would read."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200.layer import Vsa2Layer

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("projection", ["int8", "fp8"])
def test_what_a_layer_holds_between_calls(projection):
    p = vb.make_params(1, 2, 2, 64, (4, 8, 8), select_mode=vb.PER_QUERY, topk=2)
    layer = Vsa2Layer(p, 256, (16, 24, 24), projection=projection)
    gen = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(BF)
    layer.set_weights(randn(layer.width, 256) / 16, randn(256, 2) / 16, None, None)
    x = randn(1, layer.tokens, 256)
    first = layer.forward(x).clone()          # (and what the attention makes once)
    again = layer.forward(x)
    assert torch.equal(again, first)
    del again
    if projection == "int8":
        layer.saved = None
    before = torch.cuda.memory_allocated()
    for _ in range(2):
        layer.forward(x)
        if projection == "int8":
            assert torch.cuda.memory_allocated() == before and layer.saved is None
        else:
            layer.backward(first)             # (one that trains holds them: backward works)
    if projection == "int8":
        with pytest.raises(RuntimeError, match="no backward"):
            layer.backward(first)
