"""What lies behind the columns of a bf16 result in its rows stays as it is, also where the rows begin on 16-byte boundaries and n does not end on one (tensor copies write whole units of 16 bytes)."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from test_gpu_fp8_kernels import product, whole_numbers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(1, 5, 6), (20, 37, 128), (4, 533, 110), (40, 613, 44), (100, 61, 510), (1095, 197, 42), (300, 8190, 512), (2050, 4609, 200), (256, 9677, 512),
                                   (509, 6243, 648), (511, 15351, 640), (8400, 2303, 100), (200, 75, 3000), (97, 131, 5000), (1536, 637, 20000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_longer_than_the_result(m, n, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(m + n + k)
    a, b = whole_numbers(gen, m, k, 1), whole_numbers(gen, n, k, 1)
    ws, want = vb.fp8_matmul_workspace(m, n, k), product(a, b).to(dtype)
    ld = -(-n // 8) * 8 + 8
    room = torch.full((m + 2, ld), float("nan"), dtype=dtype, device="cuda")
    c = room[1:m + 1, :n]
    vb.vsa2_fp8_matmul(a, b, c, ws)
    assert torch.equal(c, want)
    assert room[:, n:].isnan().all() and room[0].isnan().all() and room[m + 1].isnan().all()


def test_two_results_side_by_side():
    """A result in the first columns of rows that hold another one behind it."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    a, b = whole_numbers(gen, 300, 400, 1), whole_numbers(gen, 1000, 400, 1)
    ws, want = vb.fp8_matmul_workspace(300, 1000, 400), product(a, b).bfloat16()
    rows = torch.empty(300, 1000, dtype=torch.bfloat16, device="cuda")
    first, second = vb.Fp8(b.values[:603], b.scales[:, :603].contiguous()), vb.Fp8(b.values[603:], b.scales[:, 603:].contiguous())
    vb.vsa2_fp8_matmul(a, second, rows[:, 603:], ws)
    vb.vsa2_fp8_matmul(a, first, rows[:, :603], ws)
    assert torch.equal(rows, want)
