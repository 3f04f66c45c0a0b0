"""Quantisation of blocks that hold infinities and NaN, in every kernel: rows alone and tiles, blocks of 128 and of 128 x 128, rows on 16-byte boundaries and off them."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from test_gpu_fp8 import check_form

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


def matrix(rows, cols, dtype, seed):
    """Random values with one to all of a block's not finite here and there: at its ends, in the last part of a row, in neighbouring rows of a warp or in one of them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=gen, device="cuda"))
    odd = torch.tensor([NAN, INF, -INF], device="cuda")
    for r in range(0, rows, 3):
        c = int(torch.randint(0, cols, (1,), generator=gen, device="cuda"))
        x[r, c] = odd[r % 3]
    x[0, 0], x[rows - 1, cols - 1] = INF, NAN
    x[rows // 2, :128] = INF                                  # a block with nothing finite
    x[rows // 2, 128:256] = NAN
    x[rows // 3, -5:] = -INF
    if rows > 128:
        x[128:, :128] = odd[torch.randint(0, 3, x[128:, :128].shape, generator=gen, device="cuda")]      # a square of them
    return x.to(dtype)


@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 7), (16, 512), (33, 700), (129, 1100), (200, 513), (257, 129)])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("squares", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_blocks_with_values_that_are_not_finite(rows, cols, dtype, squares, shift):
    x = matrix(rows, cols, dtype, rows + cols)
    ld = -(-cols // 8) * 8 + shift                            # on 16-byte boundaries, or neither the first row nor their distance
    room = torch.full((shift + rows * ld + 8,), NAN, dtype=dtype, device="cuda")
    view = room[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(x)
    xt = x.T.contiguous()
    for form, form_t in ((True, False), (False, True), (True, True)):
        out, out_t = vb.Fp8.empty(rows, cols) if form else None, vb.Fp8.empty(cols, rows) if form_t else None
        vb.vsa2_fp8_quantize(view, out, out_t, squares=squares)
        if form:
            check_form(out, x, squares)
            assert torch.equal(out.values.float().isnan(), ~x.isfinite())
        if form_t:
            check_form(out_t, xt, squares)


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_row_alone_and_beside_rows_that_are_not_finite(dtype):
    """A block's values do not depend on what the rows and blocks beside it hold."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(40, 640, generator=gen, device="cuda").to(dtype)
    want = vb.Fp8.empty(40, 640)
    vb.vsa2_fp8_quantize(x, want)
    y = x.clone()
    y[::2, 128:256] = NAN
    y[::2, 300] = INF
    got = vb.Fp8.empty(40, 640)
    vb.vsa2_fp8_quantize(y, got)
    assert torch.equal(got.values[1::2].float(), want.values[1::2].float()) and torch.equal(got.scales[:, 1::2], want.scales[:, 1::2])
    for cols in (slice(0, 128), slice(384, 640)):
        assert torch.equal(got.values[::2, cols].float(), want.values[::2, cols].float())
