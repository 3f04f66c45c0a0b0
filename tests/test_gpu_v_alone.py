"""The values alone, without queries and keys, through the calls with a norm: forward and backward take a None on both sides."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inputs", [(None, None), (None, None, None)])
def test_values_alone(inputs):
    rope, v = vb.vsa2_rope_plan(64, (16, 24, 24)), torch.randn(2, 3, 24, 64, device="cuda")
    y, dx = torch.empty_like(v), torch.empty_like(v)
    vb.vsa2_qkv_fwd(rope, (None, None, v), (None, None, y), grid=(2, 3, 4))
    ws = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    dw = [torch.full((64,), 7.0, device="cuda") for _ in range(2)]
    vb.vsa2_qkv_bwd(rope, inputs, (None, None, v), (None, None, dx), None, None, *dw, ws, grid=(2, 3, 4))
    assert torch.equal(y, v) and torch.equal(dx, v)
    assert not dw[0].any() and not dw[1].any()          # sums over nothing


def test_inputs_missing_for_a_gradient_that_is_given():
    rope, g = vb.vsa2_rope_plan(64, (16, 24, 24)), torch.randn(1, 3, 24, 64, device="cuda")
    ws = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    with pytest.raises(vb.Vsa2Error) as e:
        vb.vsa2_qkv_bwd(rope, (None, None), (g, None, None), (torch.empty_like(g), None, None), None, None, None, None, ws, grid=(2, 3, 4))
    assert e.value.code == vb.ERR_INVALID_ARG
