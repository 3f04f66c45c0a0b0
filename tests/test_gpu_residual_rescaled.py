"""Backward of rows whose mean square is far from one, which are taken again times a power of two: all three gradients, in every kernel form, against the formulas in 64 bits."""
import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
# as in the tests of ordinary rows: what fp32 leaves of a normed row, here of up to 20,011 elements
FINE = 2.0 ** -18


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def check(size, eps, cols, stream_type, rows, with_dh):
    gen = torch.Generator(device="cuda").manual_seed(cols + rows)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    h = (randn(rows, cols).clamp(-3, 3) * size).to(stream_type)
    r = float((1 / torch.sqrt((h.double() ** 2).mean(dim=1) + eps)).max())
    dy = randn(rows, cols).to(BF)
    dh = (randn(rows, cols) * r).to(stream_type) if with_dh else None      # of the size of what the norm passes on
    w = 1 + 0.1 * randn(cols)
    dr, dx, dw = torch.empty_like(h), torch.empty(rows, cols, device="cuda"), torch.full((cols,), float("nan"), device="cuda")
    ws = torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    p = 0.2
    vb.vsa2_residual_norm_bwd(h, dy, dh, w, eps=eps, d_residual=dr, dx=dx, d_weight=dw, workspace=ws, p=p, rng=torch.tensor([9, 8], device="cuda"))
    d, want_w, terms, terms_w = ref.gradients(h, dy, dh, w, eps)
    factor = ref.factors(9, 8, rows, cols, p).cuda()
    # (2^-126 / 2^24: a step of subnormal numbers, where gradients of large rows end)
    assert ((dr.double() - d).abs() <= 2 * FINE * terms + half_step(stream_type) * d.abs() + 2.0 ** -126 * half_step(stream_type)).all()
    assert ((dx.double() - d * factor).abs() <= (2 * FINE * terms + 2.0 ** -23 * d.abs()) * factor + 2.0 ** -148).all()
    # a column's terms are added one behind the other in a CTA and then over the CTAs: as in the test of ordinary rows
    assert ((dw.double() - want_w).abs() <= (FINE + 2.0 ** -16) * terms_w + 1e-37).all()


SIZES = [(1e-30, 0.0), (1e-20, 0.0), (1e-12, 0.0), (1e12, 0.0), (1e19, 0.0), (1e30, 0.0), (1e12, 1e-6), (1e30, 1e-6), (1e-20, 1e-30), (1e-15, 1e-30), (1e-12, 1e-30), (1.0, 0.0)]


@pytest.mark.parametrize("size,eps", SIZES)
@pytest.mark.parametrize("cols", [7, 64, 1536, 1531, 4608, 5003, 8192, 20000, 20011])
@pytest.mark.parametrize("stream_type", [BF, F])
def test_gradients_of_rows_of_one_size(size, eps, cols, stream_type):
    check(size, eps, cols, stream_type, 3, True)
    check(size, eps, cols, stream_type, 1, False)


@pytest.mark.parametrize("stream_type", [BF, F])
@pytest.mark.parametrize("cols", [1536, 9000])
def test_more_rows_than_the_device_holds_at_a_time(stream_type, cols):
    """The next row is on its way while one is taken again."""
    check(1e-20, 0.0, cols, stream_type, 2000, True)
    check(1e20, 1e-6, cols, stream_type, 2000, False)


def test_rows_of_all_sizes_beside_one_another():
    """A row that is taken again changes nothing of the rows before and behind it: the same bits as alone; the weight's gradient from rows of every size."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows, cols = 4000, 1536
    h = torch.randn(rows, cols, generator=gen, device="cuda")
    scale = torch.tensor([1.0, 1e-15, 1.0, 1e18], device="cuda").repeat(rows // 4).unsqueeze(1)
    h = h * scale
    dy = torch.randn(rows, cols, generator=gen, device="cuda").to(BF)
    dr, dw = torch.empty_like(h), torch.empty(cols, device="cuda")
    ws = torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    vb.vsa2_residual_norm_bwd(h, dy, eps=0.0, d_residual=dr, d_weight=dw, workspace=ws)
    d, want_w, terms, terms_w = ref.gradients(h, dy, None, None, 0.0)
    assert ((dr.double() - d).abs() <= 2 * FINE * terms + 2.0 ** -24 * d.abs()).all()
    assert ((dw.double() - want_w).abs() <= (FINE + 2.0 ** -16) * terms_w).all()
    for at in (0, 1, 2, 3, 1997, rows - 1):
        one = torch.empty(1, cols, device="cuda")
        vb.vsa2_residual_norm_bwd(h[at:at + 1], dy[at:at + 1], eps=0.0, d_residual=one)
        assert torch.equal(one[0], dr[at])
