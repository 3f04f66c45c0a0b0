"""GPU parity of the quantisation to whole numbers and of their product."""
import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 5120), (5, 15), (3, 129), (257, 1000), (64, 2047), (130, 4600), (2, 16384), (3, 16391), (2, 131071), (2, 300000)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_quantized_rows(rows, cols, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    x = (torch.randn(rows, cols, generator=gen, device="cuda") * torch.exp(3 * torch.randn(rows, 1, generator=gen, device="cuda"))).to(dtype)
    out = vb.Int8.empty(rows, cols)
    vb.vsa2_int8_quantize(x, out)
    q, m, _ = ref.int8_of(x.float())
    assert torch.equal(out.values, q)
    assert ((out.scales.double() - m.double() / 127).abs() <= 2.0 ** -24 * m.double() / 127).all()
    assert ((out.dequantize() - x.float()).abs() <= m.unsqueeze(1) / 127 * (0.5 + 2.0 ** -14)).all()


def test_extreme_rows():
    x = torch.zeros(9, 200, device="cuda")
    x[1] = 3.4e38
    x[2, 5] = 1e-40
    x[3, 7], x[3, 8] = float("inf"), 1.0
    x[4, 199] = float("nan")
    x[5, 0], x[5, 1], x[5, 2], x[5, 3] = 127.0, 0.5, 1.5, -2.5      # ties go to even
    x[6, 0], x[6, 1] = -1e-30, 2e-31
    x[7, 0], x[7, 1] = float("-inf"), float("nan")
    out = vb.Int8.empty(9, 200)
    vb.vsa2_int8_quantize(x, out)
    assert not out.values[0].any() and out.scales[0] > 0
    assert (out.values[1] == 127).all() and abs(float(out.scales[1]) / (3.4e38 / 127) - 1) < 1e-6
    assert not out.values[2].any() and out.scales[2].isfinite()
    for row in (3, 4, 7):
        assert out.scales[row].isnan() and not out.values[row].any()
    assert out.values[5, :4].tolist() == [127, 0, 2, -2] and out.scales[5] == 1
    assert out.values[6, :2].tolist() == [-127, 25]


def test_strided_and_misaligned_rows():
    gen = torch.Generator(device="cuda").manual_seed(2)
    for dtype in (BF, F):
        room = torch.randn(70, 701, generator=gen, device="cuda").to(dtype)
        x = room[:, 3:603]
        wide = torch.full((70, 640), 5, dtype=torch.int8, device="cuda")
        out = vb.Int8(wide[:, :600], torch.empty(70, device="cuda"))
        vb.vsa2_int8_quantize(x, out)
        assert torch.equal(out.values, ref.int8_of(x.float())[0]) and (wide[:, 600:] == 5).all()


# ------------------------------------------------------------------------------------------------------------- product
def operand(gen, rows, cols, extreme=False):
    f = vb.Int8.empty(rows, cols)
    f.values.copy_(torch.randint(-128, 128, (rows, cols), generator=gen, device="cuda"))
    if extreme:
        f.values.fill_(-128)
    f.scales.copy_(torch.exp(torch.randn(rows, generator=gen, device="cuda")) * 1e-2)
    return f


def expected(a, b, bias, dtype):
    """The sum exactly (fp64 holds it), to fp32, times a's scale, then times b's plus the bias with one rounding.  (fp64 holds the product of two fp32 numbers; with a bias the sum is
    rounded to fp64 first, which changes the fp32 result once in 2^29.)"""
    total = a.values.double() @ b.values.double().T
    t = total.float() * a.scales.unsqueeze(1)
    y = t.double() * b.scales.double()
    return (y if bias is None else y + bias.double()).float().to(dtype)


SHAPES = [
    (1, 1, 1), (1, 128, 128), (1, 15, 600), (2, 1000, 129), (7, 130, 1024), (32, 200, 4100), (5, 19200, 1000), (1, 1536, 131071),
    (33, 128, 130), (200, 72, 3000), (5200, 120, 130), (5204, 3, 2216), (128, 512, 128), (97, 136, 5000), (256, 4608, 640), (700, 904, 1100),
    (129, 256, 200), (1000, 264, 3000), (300, 8192, 512), (4096, 4608, 640), (4093, 4616, 136), (1536, 640, 20000), (2978, 488, 17078),
    (20000, 4608, 128), (8400, 2304, 100), (256, 9680, 512), (512, 15360, 640), (511, 15352, 640), (509, 6240, 648), (505, 6248, 1200), (250, 16576, 1000),
    (130, 257, 640), (225, 300, 75), (300, 515, 1153), (449, 2304, 512),
    # more of tiles of 32 and 128 columns: all ranges of K in one, ragged and on the edge, results on 16-byte boundaries and off them; groups of tiles and a shorter last one
    (9, 4608, 100), (32, 19200, 1536), (31, 4603, 128), (17, 40, 640), (33, 96, 128), (700, 64, 100), (9000, 128, 256), (64, 4608, 1536), (128, 15360, 640), (100, 9000, 512),
    (20000, 264, 128), (40000, 520, 64), (2025, 4603, 1530), (3000, 1536, 1536), (200, 71, 100), (4000, 125, 256),
    # pairs on tiles of 128 columns, whole and in ranges of K
    (892, 1328, 6331), (3965, 259, 7192), (1214, 512, 6515), (155, 2025, 8135), (2810, 248, 7641),
]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [F, BF])
def test_products(m, n, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(m + 3 * n + 7 * k)
    a, b = operand(gen, m, k), operand(gen, n, k)
    bias = torch.randn(n, generator=gen, device="cuda")
    c = torch.empty(m, n, dtype=dtype, device="cuda")
    ws = vb.int8_matmul_workspace(m, n, k)
    for _ in range(2):
        c.fill_(float("nan"))
        vb.vsa2_int8_matmul(a, b, c, ws)
        want = expected(a, b, None, dtype)
        assert torch.equal(c, want), int((c != want).sum())
    vb.vsa2_int8_matmul(a, b, c, ws, bias=bias)
    want = expected(a, b, bias, dtype)
    step = 2.0 ** -23 if dtype == F else 2.0 ** -7      # (one step where the two roundings of the expectation fall badly)
    assert ((c.double() - want.double()).abs() <= step * want.double().abs()).all() and (c != want).double().mean() < 1e-4
    assert vb.vsa2_device_status(ws) == vb.OK


@pytest.mark.parametrize("m,n,k", [(9, 4608, 100), (100, 264, 3000), (33, 96, 128), (700, 64, 100), (300, 8192, 512), (1536, 640, 20000), (5, 4608, 1536)])
@pytest.mark.parametrize("skip", [0, 1])
def test_every_kernel_with_results_on_and_off_boundaries(m, n, k, skip):
    """bf16 with rows of 16-byte units: tensor copies, and plain stores where the first result is off; nothing else is written."""
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    a, b, bias = operand(gen, m, k), operand(gen, n, k), torch.randn(n, generator=gen, device="cuda")
    room = torch.full((m, n + 16), 7.0, dtype=BF, device="cuda")
    vb.vsa2_int8_matmul(a, b, room[:, skip:skip + n], vb.int8_matmul_workspace(m, n, k), bias=bias)
    want = expected(a, b, bias, BF)
    got = room[:, skip:skip + n]
    assert ((got.double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs()).all() and (got != want).double().mean() < 1e-4
    assert (room[:, :skip] == 7).all() and (room[:, skip + n:] == 7).all()


@pytest.mark.parametrize("m", [1, 2, 3, 4, 7, 8, 9])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 1000])
@pytest.mark.parametrize("k", [1, 15, 16, 17, 63, 64, 65, 500, 512, 2561, 5120])
def test_few_rows(m, n, k):
    gen = torch.Generator(device="cuda").manual_seed(m + 3 * n + 7 * k)
    a, b = operand(gen, m, k), operand(gen, n, k)
    bias = torch.randn(n, generator=gen, device="cuda")
    room = torch.full((m, n + 3), 7.0, device="cuda")
    ws = vb.int8_matmul_workspace(m, n, k)
    vb.vsa2_int8_matmul(a, b, room[:, 1:1 + n], ws)
    assert torch.equal(room[:, 1:1 + n], expected(a, b, None, F)) and (room[:, 0] == 7).all() and (room[:, 1 + n:] == 7).all()
    c = torch.empty(m, n, dtype=BF, device="cuda")
    vb.vsa2_int8_matmul(a, b, c, ws, bias=bias)
    want = expected(a, b, bias, BF)
    assert ((c.double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs()).all()


@pytest.mark.parametrize("m,n,k", [(3, 200, 131071), (300, 600, 131071)])
def test_the_largest_sums(m, n, k):
    gen = torch.Generator(device="cuda").manual_seed(1)
    a, b = operand(gen, m, k, extreme=True), operand(gen, n, k, extreme=True)
    c, ws = torch.empty(m, n, device="cuda"), vb.int8_matmul_workspace(m, n, k)
    vb.vsa2_int8_matmul(a, b, c, ws)
    assert torch.equal(c, expected(a, b, None, F))


@pytest.mark.parametrize("pad,skip,n", [(8, 0, 520), (3, 0, 520), (8, 1, 520), (0, 0, 513), (5, 2, 300)])
@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("m", [3, 100, 600])
def test_results_of_any_stride_and_address(pad, skip, n, dtype, m):
    gen = torch.Generator(device="cuda").manual_seed(n + pad)
    k = 333
    va = torch.randint(-128, 128, (m, 352), generator=gen, device="cuda").to(torch.int8)
    a, b = vb.Int8(va[:, :k], torch.rand(m, generator=gen, device="cuda")), operand(gen, n, k)
    room = torch.full((m, n + pad + skip), 7.0, dtype=dtype, device="cuda")
    vb.vsa2_int8_matmul(a, b, room[:, skip:skip + n], vb.int8_matmul_workspace(m, n, k))
    assert torch.equal(room[:, skip:skip + n], expected(a, b, None, dtype))
    assert (room[:, :skip] == 7).all() and (room[:, skip + n:] == 7).all()


def test_a_row_alone_and_among_others_has_the_same_bits():
    gen = torch.Generator(device="cuda").manual_seed(4)
    m, n, k = 600, 1536, 1536
    a, b, bias = operand(gen, m, k), operand(gen, n, k), torch.randn(1536, generator=gen, device="cuda")
    ws = vb.int8_matmul_workspace(m, n, k)
    whole = torch.empty(m, n, dtype=BF, device="cuda")
    vb.vsa2_int8_matmul(a, b, whole, ws, bias=bias)
    for rows in ([5], [0, 599], list(range(100)), list(range(300))):
        part = vb.Int8.empty(len(rows), k)
        part.values.copy_(a.values[rows])
        part.scales.copy_(a.scales[rows])
        c = torch.empty(len(rows), n, dtype=BF, device="cuda")
        vb.vsa2_int8_matmul(part, b, c, ws, bias=bias)
        assert torch.equal(c, whole[rows])


def test_rows_without_a_scale_are_nan_and_sums_over_nothing_are_the_bias():
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(40, 300, generator=gen, device="cuda")
    x[7, 3] = float("inf")
    a, b = vb.Int8.empty(40, 300), operand(gen, 200, 300)
    vb.vsa2_int8_quantize(x, a)
    c, ws = torch.empty(40, 200, device="cuda"), vb.int8_matmul_workspace(40, 200, 300)
    vb.vsa2_int8_matmul(a, b, c, ws)
    assert c[7].isnan().all() and c.isnan().sum() == 200
    bias = torch.randn(200, generator=gen, device="cuda")
    for m in (0, 3):
        c = torch.full((m, 200), 9.0, device="cuda")
        vb.vsa2_int8_matmul(vb.Int8.empty(m, 0), vb.Int8.empty(200, 0), c, ws, bias=bias)
        assert (c == bias).all()
        vb.vsa2_int8_matmul(vb.Int8.empty(m, 0), vb.Int8.empty(200, 0), c, ws)
        assert (c == 0).all()
    vb.vsa2_int8_matmul(vb.Int8.empty(3, 64), vb.Int8.empty(0, 64), torch.empty(3, 0, device="cuda"), ws)


def test_one_workspace_serves_smaller_products():
    gen = torch.Generator(device="cuda").manual_seed(6)
    ws = vb.int8_matmul_workspace(2000, 1024, 9000)
    for m, n, k in ((2000, 1024, 9000), (40, 1000, 9000), (1500, 640, 8000), (300, 130, 5000), (1, 1024, 9000)):
        a, b = operand(gen, m, k), operand(gen, n, k)
        c = torch.empty(m, n, device="cuda")
        vb.vsa2_int8_matmul(a, b, c, ws)
        assert torch.equal(c, expected(a, b, None, F))
