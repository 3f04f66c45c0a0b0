"""How much of a long sum one truncating accumulator of the tensor cores may hold before an fp32 result adds it up."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blocks", [40, 41, 64, 96, 130])
def test_a_large_product_swallows_the_rest_of_its_own_piece_alone(blocks):
    """The first product is 2^24, every 32 values behind it sum to 0.5, a quarter of the accumulator's last place there: lost where they meet it.  An fp32 result is summed in
    pieces of 40 blocks of 128, so what is missing is at most the 39 blocks (2 each) behind the large product in its piece, and a unit (2) for the pieces' additions; what lies
    in later pieces is there.  1400 x 2300 has tiles for all SMs, so K is not cut into ranges."""
    m, n, k = 1400, 2300, 128 * blocks
    a, b = vb.Fp8.empty(m, k), vb.Fp8.empty(n, k)
    va, vb_ = torch.zeros(1, k, device="cuda"), torch.zeros(1, k, device="cuda")
    va[0, 0] = vb_[0, 0] = 1.0
    va[0, 128::32], vb_[0, 128::32] = 1.0, 0.5
    for f, v in ((a, va), (b, vb_)):
        f.values.copy_(v.to(torch.float8_e4m3fn).expand(f.shape[0], k))
        f.scales.fill_(127)
        f.scales[0, :, 0] = 127 + 12
    ws, c = vb.fp8_matmul_workspace(m, n, k), torch.empty(m, n, device="cuda")
    vb.vsa2_fp8_matmul(a, b, c, ws)
    exact = 2.0 ** 24 + 2.0 * (blocks - 1)
    missing = exact - c.double()
    assert float(missing.max()) <= 2.0 * 39 + 2.0 and float(missing.min()) >= -2.0, (float(missing.min()), float(missing.max()))
