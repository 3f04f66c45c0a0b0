"""Tensors of more than 2^31 elements: the last rows as the same rows alone."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from test_gpu_fp8_kernels import product

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("squares", [False, True])
def test_quantisation(squares):
    rows, cols = 128 * 3500, 4808                         # 2.15e9 elements; the transpose's rows end beyond 2^31 too
    x = torch.empty(rows, cols, dtype=BF, device="cuda")
    x[:128].normal_()
    for r in range(128, rows, 128 * 500):
        x[r:r + 128 * 500] = 1.5
    x[-256:].normal_()
    out, out_t = vb.Fp8.empty(rows, cols), vb.Fp8.empty(cols, rows)
    vb.vsa2_fp8_quantize(x, out, out_t, squares=squares)
    alone = vb.Fp8.empty(rows, cols)
    if not squares:
        vb.vsa2_fp8_quantize(x, alone)                    # (the rows' own kernel)
        assert torch.equal(alone.values[-256:].float(), out.values[-256:].float()) and torch.equal(alone.scales, out.scales)
    del alone
    for part in (slice(0, 128), slice(rows - 256, rows)):
        want, want_t = vb.Fp8.empty(part.stop - part.start, cols), vb.Fp8.empty(cols, part.stop - part.start)
        vb.vsa2_fp8_quantize(x[part], want, want_t, squares=squares)
        assert torch.equal(out.values[part].float(), want.values.float()) and torch.equal(out.scales[:, part], want.scales)
        assert torch.equal(out_t.values[:, part].float(), want_t.values.float())


def whole(gen, rows, cols, tail):
    """Ones, and in the last rows small whole numbers."""
    f = vb.Fp8.empty(rows, cols)
    f.values.view(torch.uint8).fill_(0x38)                # 1.0
    f.values[-tail:] = torch.randint(-2, 3, (tail, cols), generator=gen, device="cuda", dtype=torch.int8).to(BF).to(torch.float8_e4m3fn)
    f.scales.fill_(127)
    return f


@pytest.mark.parametrize("m,n,k,dtype", [(140000, 15368, 128, BF), (140000, 15371, 128, BF), (140000, 15368, 128, torch.float32), (270000, 136, 8192, BF)])
def test_products(m, n, k, dtype):
    """Results of more than 2^31 elements, and an operand of more than 2^31 bytes."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    a, b = whole(gen, m, k, 300), whole(gen, n, k, min(n, 300))
    c, ws = torch.empty(m, n, dtype=dtype, device="cuda"), vb.fp8_matmul_workspace(m, n, k)
    vb.vsa2_fp8_matmul(a, b, c, ws)
    for rows in (slice(0, 100), slice(m - 300, m)):
        want = product(vb.Fp8(a.values[rows], a.scales[:, rows].contiguous()), b)
        assert torch.equal(c[rows], want.to(dtype))
    assert vb.vsa2_device_status(ws) == vb.OK


def test_norms_rotation_and_heads():
    grid, n, batch, hq, hk, dim = (21, 45, 80), 75600, 2, 40, 34, 128
    n_heads = hq + 2 * hk
    rope = vb.vsa2_rope_plan(dim, (44, 42, 42))
    packed = torch.empty(batch, n + 6000, n_heads, dim, dtype=BF, device="cuda")      # (rows of a longer buffer: the last ones begin beyond 2.17e9 elements)
    packed.fill_(0.5)
    packed[:, n - 64:].normal_()
    x = packed[:, :n].transpose(1, 2)
    x = (x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:])
    w = [torch.linspace(0.5, 1.5, dim, device="cuda") for _ in range(2)]
    y = [torch.empty(batch, h, n, dim, dtype=BF, device="cuda") for h in (hq, hk, hk)]
    vb.vsa2_qkv_fwd(rope, x, y, *w, grid=grid)
    part = [v[:, :, n - 64:] for v in x]
    want = [torch.empty(batch, h, 64, dim, dtype=BF, device="cuda") for h in (hq, hk, hk)]
    vb.vsa2_qkv_fwd(rope, part, want, *w, grid=grid, first=n - 64)
    assert all(torch.equal(a[:, :, n - 64:], b) for a, b in zip(y, want))
    dx = torch.zeros_like(packed)
    d = dx[:, :n].transpose(1, 2)
    ws = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(dim), dtype=torch.uint8, device="cuda")
    vb.vsa2_qkv_bwd(rope, x, y, (d[:, :hq], d[:, hq:hq + hk], d[:, hq + hk:]), *w, None, None, ws, grid=grid)
    got = [torch.empty(batch, h, 64, dim, dtype=BF, device="cuda") for h in (hq, hk, hk)]
    vb.vsa2_qkv_bwd(rope, part, want, got, *w, None, None, ws, grid=grid, first=n - 64)
    assert all(torch.equal(a, b) for a, b in zip((d[:, :hq, n - 64:], d[:, hq:hq + hk, n - 64:], d[:, hq + hk:, n - 64:]), got))
    assert not dx[:, n:].any()
