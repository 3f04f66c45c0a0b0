"""Every kernel of the 8-bit product (fp8_shapes) on small whole numbers, whose sums fit 24 bits: any order of the additions gives the same fp32 value, so results are compared exactly."""
import pytest
import torch

from fp8_shapes import SHAPES
from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def whole_numbers(gen, rows, cols, scales):
    """Values -2 .. 2; scales one or two, different from block to block.  (20,000 products of at most 16: below 2^19.)"""
    f = vb.Fp8.empty(rows, cols)
    f.values.copy_(torch.randint(-2, 3, (rows, cols), generator=gen, device="cuda", dtype=torch.int8).to(BF).to(torch.float8_e4m3fn))
    f.scales.copy_(torch.randint(127, 127 + scales, f.scales.shape, generator=gen, device="cuda", dtype=torch.uint8))
    return f


def product(a, b):
    return (a.dequantize().double() @ b.dequantize().double().T).float()


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_every_kernel(m, n, k):
    gen = torch.Generator(device="cuda").manual_seed(m + 3 * n + 7 * k)
    a, b = whole_numbers(gen, m, k, 2), whole_numbers(gen, n, k, 2)
    want, ws = product(a, b), vb.fp8_matmul_workspace(m, n, k)
    # rows 1 .. m of a larger matrix: on 16-byte boundaries where n is a multiple of 8, off them with an odd row stride, fp32
    for dtype, extra in ((BF, 8), (BF, 3), (F, 8)):
        room = torch.full((m + 2, n + extra), float("nan"), dtype=dtype, device="cuda")
        c = room[1:m + 1, :n]
        vb.vsa2_fp8_matmul(a, b, c, ws)
        assert torch.equal(c, want.to(dtype)), int((c != want.to(dtype)).sum())
        assert room[0].isnan().all() and room[m + 1].isnan().all() and room[:, n:].isnan().all()
    assert vb.vsa2_device_status(ws) == vb.OK


@pytest.mark.parametrize("m,n,k", [(256, 9680, 512), (300, 8192, 512), (129, 264, 1000), (20, 1160, 600)])
def test_scales_of_every_row_and_block(m, n, k):
    """Scales from 2^-20 to 2^20 and from 2^-3 to 2^3, one value not zero in each row's block: every element is one product, or a few far apart, and exact in fp32 where it is one."""
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    a, b = vb.Fp8.empty(m, k), vb.Fp8.empty(n, k)
    va = torch.zeros(m, k, device="cuda")
    at = torch.randint(0, k, (m,), generator=gen, device="cuda")          # a row of A picks one column of K
    va[torch.arange(m, device="cuda"), at] = 1.0
    a.values.copy_(va.to(torch.float8_e4m3fn))
    b.values.copy_(torch.randint(-8, 9, (n, k), generator=gen, device="cuda").float().to(torch.float8_e4m3fn))
    a.scales.copy_(torch.randint(127 - 20, 127 + 21, a.scales.shape, generator=gen, device="cuda", dtype=torch.uint8))
    b.scales.copy_(torch.randint(127 - 3, 127 + 4, b.scales.shape, generator=gen, device="cuda", dtype=torch.uint8))
    want, ws = product(a, b), vb.fp8_matmul_workspace(m, n, k)
    for dtype in (F, BF):
        c = torch.empty(m, n, dtype=dtype, device="cuda")
        vb.vsa2_fp8_matmul(a, b, c, ws)
        assert torch.equal(c, want.to(dtype))


def test_values_of_normal_numbers_on_swapped_operands():
    """A result of tiles with A's rows as lanes against 64 bits: each of the k / 32 additions to an accumulator may lose 2^-23 of it, at most the sum of the magnitudes; half a unit of
    bf16's last place on top."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    m, n, k = 511, 15352, 640
    assert vb.vsa2_debug_fp8_matmul_plan(m, n, k)[2] == 1
    a, b = vb.Fp8.empty(m, k), vb.Fp8.empty(n, k)
    vb.vsa2_fp8_quantize(torch.randn(m, k, generator=gen, device="cuda").to(BF), a)
    vb.vsa2_fp8_quantize((torch.randn(n, k, generator=gen, device="cuda") * k ** -0.5).to(BF), b, squares=True)
    c, ws = torch.empty(m, n, dtype=BF, device="cuda"), vb.fp8_matmul_workspace(m, n, k)
    vb.vsa2_fp8_matmul(a, b, c, ws)
    A, B = a.dequantize().double(), b.dequantize().double()
    want, size = A @ B.T, A.abs() @ B.abs().T
    bound = (k / 32 + 8) * 2.0 ** -23 * size
    bound = bound + torch.ldexp(torch.ones_like(want), torch.frexp(want.abs() + bound)[1] - 9)
    assert ((c.double() - want).abs() <= bound).all()
    again = torch.empty_like(c)
    vb.vsa2_fp8_matmul(a, b, again, ws)
    assert torch.equal(c, again)
