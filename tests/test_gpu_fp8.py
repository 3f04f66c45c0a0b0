"""GPU parity of the 8-bit quantisation and product against their definitions in 64 bits."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def reference_scales(x, squares):
    """Exponents of the blocks [rows, blocks] in 64 bits: the least e >= -127 with max|x| <= 448 2^e over the finite values."""
    rows, cols = x.shape
    a = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).abs().double()
    blocks = [a[:, c:c + 128].amax(1) for c in range(0, cols, 128)]
    top = torch.stack(blocks, 1)
    if squares:
        top = torch.cat([top[r:r + 128].amax(0, keepdim=True).expand(min(128, rows - r), -1) for r in range(0, rows, 128)])
    e = torch.full_like(top, -127)
    for _ in range(2):      # a start from the logarithm, then exact comparisons
        e = torch.maximum(torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)) - 1, e), torch.full_like(e, -127))
    for _ in range(3):
        e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    return e


def check_form(form, x, squares):
    """Scales exactly, values exactly the rounding of x / 2^e (by torch's conversion of the fp32 quotient, which is exact)."""
    rows, cols = x.shape
    e = reference_scales(x, squares)
    got = form.scales.transpose(0, 1).reshape(rows, -1)
    assert torch.equal(got[:, :e.shape[1]].double() - 127, e)
    assert not got[:, e.shape[1]:].any()
    scaled = x.double() / torch.exp2(e).repeat_interleave(128, 1)[:, :cols]
    want = torch.where(torch.isfinite(x), scaled.float(), torch.full_like(x, float("nan"), dtype=F)).to(torch.float8_e4m3fn).float()
    same = (form.values.float() == want) | (form.values.float().isnan() & want.isnan())
    assert same.all(), int((~same).sum())


SIZES = [(1, 1), (1, 128), (3, 129), (128, 512), (130, 513), (257, 1000), (16, 2047), (1000, 77), (129, 4600), (64, 15)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("squares", [False, True])
def test_quantized_forms(rows, cols, dtype, squares):
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda") * torch.exp(3 * torch.randn(rows, 1, generator=gen, device="cuda"))
    x = x.to(dtype)
    forms = vb.Fp8.empty(rows, cols), vb.Fp8.empty(cols, rows)
    for f in forms:
        f.scales.fill_(99)
    vb.vsa2_fp8_quantize(x, *forms, squares=squares)
    check_form(forms[0], x, squares)
    check_form(forms[1], x.T.contiguous(), squares)
    for k in range(2):                                    # each form alone
        alone = vb.Fp8.empty(*forms[k].shape)
        vb.vsa2_fp8_quantize(x, alone if k == 0 else None, alone if k == 1 else None, squares=squares)
        assert torch.equal(alone.values.float(), forms[k].values.float()) and torch.equal(alone.scales, forms[k].scales)


def test_blocks_of_zeros_extremes_and_what_is_not_finite():
    x = torch.zeros(8, 640, device="cuda")
    x[1, :128] = 448.0                                    # the largest value itself: scale one
    x[2, 0] = 448.00003                                   # the next fp32 value: scale two
    x[3, 0], x[3, 1] = 3.0e38, -1.0                       # a scale near the top, its neighbour vanishes
    x[4, 0] = 1e-40                                       # a subnormal: the least scale
    x[5, 0], x[5, 1], x[5, 2] = float("inf"), 2.0, float("-inf")
    x[6, 130] = float("nan")
    x[7, 512:] = 1e-38
    out, out_t = vb.Fp8.empty(8, 640), vb.Fp8.empty(640, 8)
    vb.vsa2_fp8_quantize(x, out, out_t)
    check_form(out, x, False)
    check_form(out_t, x.T.contiguous(), False)
    assert out.scales[0, 1, 0] == 127 and out.scales[0, 2, 0] == 128 and out.scales[0, 0, 0] == 0
    assert out.values[5].float()[:3].isnan().tolist() == [True, False, True]


def test_strided_and_misaligned_rows():
    gen = torch.Generator(device="cuda").manual_seed(2)
    room = torch.randn(70, 701, generator=gen, device="cuda").to(BF)
    x = room[:, 3:603]                                    # rows of 1402 bytes, begun at byte 6
    out, out_t = vb.Fp8.empty(70, 600), vb.Fp8.empty(600, 70)
    vb.vsa2_fp8_quantize(x, out, out_t)
    check_form(out, x.contiguous(), False)
    check_form(out_t, x.T.contiguous(), False)
    wide = torch.full((70, 640), 5.0, device="cuda").to(torch.float8_e4m3fn)      # values beyond the columns stay
    vb.vsa2_fp8_quantize(x, vb.Fp8(wide[:, :600], out.scales))
    assert torch.equal(wide[:, :600].float(), out.values.float()) and (wide[:, 600:].float() == 5.0).all()


# ------------------------------------------------------------------------------------------------------------- product
def whole_numbers(gen, rows, cols, low_scale, high_scale):
    """A matrix whose values are small whole numbers and whose scales are different powers of two from block to block."""
    f = vb.Fp8.empty(rows, cols)
    f.values.copy_(torch.randint(-2, 3, (rows, cols), generator=gen, device="cuda").float().to(torch.float8_e4m3fn))
    f.scales.copy_(torch.randint(127 + low_scale, 128 + high_scale, f.scales.shape, generator=gen, device="cuda").to(torch.uint8))
    return f


SHAPES = [(1, 1, 1), (1, 128, 128), (1, 15, 600), (2, 1000, 129), (7, 130, 1024), (16, 256, 384), (17, 640, 5120), (33, 129, 513), (64, 384, 512),
          (65, 100, 2000), (128, 128, 128), (130, 257, 640), (225, 300, 75), (300, 515, 1153), (449, 2304, 512), (1000, 1000, 1000), (2048, 2304, 256)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [F, BF])
def test_products_of_whole_numbers_are_exact(m, n, k, dtype):
    """Every sum fits 24 bits, so any order of the additions gives the same fp32 value."""
    gen = torch.Generator(device="cuda").manual_seed(m + 3 * n + 7 * k)
    a, b = whole_numbers(gen, m, k, -1, 1), whole_numbers(gen, n, k, 0, 2)
    c = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
    ws = vb.fp8_matmul_workspace(m, n, k)
    want = (a.dequantize().double() @ b.dequantize().double().T).float().to(dtype)
    for _ in range(2):                                    # (the workspace is left as it was found)
        c.fill_(float("nan"))
        vb.vsa2_fp8_matmul(a, b, c, ws)
        assert torch.equal(c, want), int((c != want).sum())
    assert vb.vsa2_device_status(ws) == vb.OK


@pytest.mark.parametrize("m,n,k", [(1, 3200, 5120), (12, 520, 700), (100, 1536, 1536), (700, 900, 4100), (1536, 640, 20000)])
@pytest.mark.parametrize("squares", [False, True])
def test_products_of_quantized_matrices(m, n, k, squares):
    """fp32 sums: each of the k / 32 additions to an accumulator may lose 2^-23 of it (it is cut, not rounded), and an accumulator is at most the sum of the
    magnitudes; bf16 outputs add half a unit of their last place, 2^(e - 8) at 2^e."""
    gen = torch.Generator(device="cuda").manual_seed(m + n + k)
    x = torch.randn(m, k, generator=gen, device="cuda") * torch.exp(torch.randn(m, 1, generator=gen, device="cuda"))
    w = torch.randn(n, k, generator=gen, device="cuda") * k ** -0.5
    a, b = vb.Fp8.empty(m, k), vb.Fp8.empty(n, k)
    vb.vsa2_fp8_quantize(x.to(BF), a)
    vb.vsa2_fp8_quantize(w.to(BF), b, squares=squares)
    ws = vb.fp8_matmul_workspace(m, n, k)
    A, B = a.dequantize().double(), b.dequantize().double()
    want, size = A @ B.T, A.abs() @ B.abs().T
    for dtype in (F, BF):
        c = torch.empty(m, n, dtype=dtype, device="cuda")
        vb.vsa2_fp8_matmul(a, b, c, ws)
        err = (c.double() - want).abs()
        bound = (k / 32 + 8) * 2.0 ** -23 * size
        if dtype == BF:
            bound = bound + torch.ldexp(torch.ones_like(want), torch.frexp(want.abs() + bound)[1] - 9)
        assert (err <= bound).all()
        again = torch.empty_like(c)
        vb.vsa2_fp8_matmul(a, b, again, ws)
        assert torch.equal(c, again)


def test_one_workspace_serves_products_of_every_size():
    gen = torch.Generator(device="cuda").manual_seed(5)
    shapes = [(300, 515, 1153), (1, 300, 5000), (40, 700, 900), (1000, 260, 333), (3, 3, 3)]
    ws = vb.fp8_matmul_workspace(*(max(s[i] for s in shapes) for i in range(3)))
    for m, n, k in shapes * 2:
        a, b = whole_numbers(gen, m, k, 0, 1), whole_numbers(gen, n, k, 0, 1)
        c = torch.empty(m, n, dtype=F, device="cuda")
        vb.vsa2_fp8_matmul(a, b, c, ws)
        assert torch.equal(c, (a.dequantize().double() @ b.dequantize().double().T).float())


def test_nan_reaches_its_row_and_column_alone():
    gen = torch.Generator(device="cuda").manual_seed(6)
    a, b = whole_numbers(gen, 40, 300, 0, 0), whole_numbers(gen, 200, 300, 0, 0)
    ws = vb.fp8_matmul_workspace(40, 200, 300)
    c = torch.empty(40, 200, dtype=F, device="cuda")
    a.values[7, 299] = float("nan")
    b.values[130, 3] = float("nan")
    vb.vsa2_fp8_matmul(a, b, c, ws)
    bad = torch.zeros(40, 200, dtype=torch.bool, device="cuda")
    bad[7], bad[:, 130] = True, True
    assert torch.equal(c.isnan(), bad)


def test_scales_reach_from_one_end_to_the_other():
    a, b = vb.Fp8.empty(1, 128), vb.Fp8.empty(1, 128)
    for f in (a, b):
        f.values.copy_(torch.ones(1, 128, device="cuda").to(torch.float8_e4m3fn))
    ws, c = vb.fp8_matmul_workspace(1, 1, 128), torch.empty(1, 1, device="cuda")
    for ea, eb in ((0, 254), (254, 0), (247, 7), (127, 127), (60, 90)):
        a.scales.fill_(ea)
        b.scales.fill_(eb)
        vb.vsa2_fp8_matmul(a, b, c, ws)
        assert float(c) == 128.0 * 2.0 ** (ea + eb - 254)


def test_rows_of_c_may_lie_apart():
    gen = torch.Generator(device="cuda").manual_seed(7)
    a, b = whole_numbers(gen, 50, 200, 0, 1), whole_numbers(gen, 77, 200, 0, 1)
    room = torch.full((50, 101), -7.0, dtype=BF, device="cuda")
    ws = vb.fp8_matmul_workspace(50, 77, 200)
    vb.vsa2_fp8_matmul(a, b, room[:, 5:82], ws)
    assert torch.equal(room[:, 5:82], (a.dequantize().double() @ b.dequantize().double().T).to(BF))
    assert (room[:, :5] == -7).all() and (room[:, 82:] == -7).all()


def test_empty_products():
    ws = vb.fp8_matmul_workspace(4, 4, 0)
    c = torch.full((4, 4), 3.0, device="cuda")
    vb.vsa2_fp8_matmul(vb.Fp8.empty(4, 0), vb.Fp8.empty(4, 0), c, ws)
    assert not c.any()
    vb.vsa2_fp8_matmul(vb.Fp8.empty(0, 8), vb.Fp8.empty(4, 8), torch.empty(0, 4, device="cuda"), ws)
    vb.vsa2_fp8_quantize(torch.empty(0, 8, device="cuda"), vb.Fp8.empty(0, 8), vb.Fp8.empty(8, 0))


def test_graph_and_another_stream():
    gen = torch.Generator(device="cuda").manual_seed(8)
    m, n, k = 300, 515, 1153
    a, b = whole_numbers(gen, m, k, 0, 1), whole_numbers(gen, n, k, 0, 1)
    want = (a.dequantize().double() @ b.dequantize().double().T).float()
    ws, c = vb.fp8_matmul_workspace(m, n, k), torch.zeros(m, n, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    vb.vsa2_fp8_matmul(a, b, c, ws, stream=side)
    side.synchronize()
    assert torch.equal(c, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            vb.vsa2_fp8_matmul(a, b, c, ws)
    c.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c, want)


def test_long_sums_in_pieces_and_in_ranges():
    """fp32 results of more blocks of K than one accumulator sums, in few tiles (K in ranges) and in many (pieces added in place)."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    for m, n, k in ((300, 515, 20000), (5, 200, 30000), (1400, 2300, 17000), (100, 100, 33000)):
        a, b = whole_numbers(gen, m, k, 0, 1), whole_numbers(gen, n, k, 0, 1)
        want = (a.dequantize().double() @ b.dequantize().double().T).float()
        ws = vb.fp8_matmul_workspace(m, n, k)
        for dtype in (F, BF):
            c = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
            vb.vsa2_fp8_matmul(a, b, c, ws)
            assert torch.equal(c, want.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,ld", [(1, 1, 1), (3, 9, 9), (130, 131, 133), (17, 520, 527), (129, 127, 1001), (5, 513, 513)])
def test_rows_at_any_address(rows, cols, ld, dtype):
    """A matrix whose rows begin at any multiple of its type, with NaN all around it, as one on 16-byte boundaries."""
    gen = torch.Generator(device="cuda").manual_seed(21)
    x = (torch.randn(rows, cols, generator=gen, device="cuda") * 3).to(dtype)
    even = torch.zeros(rows, -(-cols // 8) * 8, dtype=dtype, device="cuda")[:, :cols]
    even.copy_(x)
    want = [vb.Fp8.empty(rows, cols), vb.Fp8.empty(cols, rows)]
    vb.vsa2_fp8_quantize(even, *want)
    alone = vb.Fp8.empty(rows, cols)
    vb.vsa2_fp8_quantize(even, alone)
    for shift in range(9):
        room = torch.full((shift + rows * ld + 16,), float("nan"), dtype=dtype, device="cuda")
        view = room[shift:shift + rows * ld].view(rows, ld)[:, :cols]
        view.copy_(x)
        got = [vb.Fp8.empty(rows, cols), vb.Fp8.empty(cols, rows)]
        vb.vsa2_fp8_quantize(view, *got)
        single = vb.Fp8.empty(rows, cols)
        vb.vsa2_fp8_quantize(view, single)
        for a, b in zip((*got, single), (*want, alone)):
            assert torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a.scales, b.scales)
