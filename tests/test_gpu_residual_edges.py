"""The residual stream's calls at the ends of their ranges: numbers at the ends of bf16, the widest rows, tensors of more than 2^31 elements, the quantiser's form from the norm."""
import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def test_sums_of_all_kinds_of_bf16_numbers():
    """h is the fp32 sum rounded, also of subnormal numbers, of numbers far apart, at overflow, and of what is not finite."""
    bits = torch.cat([torch.arange(0, 65536, 97, dtype=torch.int32), torch.tensor([0, 0x8000, 1, 0x7f, 0x80, 0x7f7f, 0xff7f, 0x7f80, 0xff80, 0x7fc0, 0x3f80, 0x3f81])])
    some = bits.to(torch.int16).view(BF).cuda()
    n = some.numel() // 8 * 8
    x = some[:n].repeat(n, 1)
    r = x.T.contiguous()
    h = torch.empty_like(x)
    vb.vsa2_residual_norm_fwd(x, r, h=h)
    want = (r.float() + x.float()).to(BF)
    same = (h == want) | (h.isnan() & want.isnan())
    assert same.all(), int((~same).sum())


@pytest.mark.parametrize("rows,cols", [(50, 1536), (50, 5120), (7, 4600), (33, 1001), (3, 20000)])
@pytest.mark.parametrize("stream_type", [BF, F])
def test_the_norm_s_form_is_the_quantiser_s(rows, cols, stream_type):
    """Values and scales are those that vsa2_fp8_quantize makes of the norm's fp32 output, bit for bit, also of rows of zeros, of padding, and of very large and small ones."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda") * torch.exp2(torch.randint(-30, 30, (rows, cols), generator=gen, device="cuda").float())
    x[1] = 0
    x[2] *= 1e-30
    x[0, cols // 2:] = 0
    x = x.to(stream_type)
    w = torch.randn(cols, generator=gen, device="cuda") * torch.exp2(torch.randint(-60, 60, (cols,), generator=gen, device="cuda").float())
    y, form, want = torch.empty(rows, cols, device="cuda"), vb.Fp8.empty(rows, cols), vb.Fp8.empty(rows, cols)
    vb.vsa2_residual_norm_fwd(x, weight=w, y=y, y_fp8=form)
    vb.vsa2_fp8_quantize(y, want)
    assert torch.equal(form.scales, want.scales)
    a, b = form.values.float(), want.values.float()
    assert ((a == b) | (a.isnan() & b.isnan())).all()


@pytest.mark.parametrize("cols", [1 << 22, (1 << 22) - 3, 200001])
def test_the_widest_rows(cols):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn(2, cols, generator=gen, device="cuda").to(BF) for _ in range(2))
    w = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
    h, y, q = torch.empty_like(r), torch.empty(2, cols, device="cuda"), vb.Int8.empty(2, cols)
    rng = torch.tensor([3, 4], device="cuda")
    vb.vsa2_residual_norm_fwd(x, r, w, h=h, y=y, y_int8=q, p=0.1, rng=rng)
    want_h = ref.stream(x, r, ref.factors(3, 4, 2, cols, 0.1))
    assert torch.equal(h, want_h)
    want, _ = ref.normed(want_h, w, 1e-6)
    # 512 threads, two pieces of eight a round: 4096 rounds of 8 steps in either of two sums at most, 2^13 steps; positive terms, whose errors of 2^-24 each are of either sign: 2^-18 with
    # a margin (2^13 steps all to one side would be 2^-12)
    assert ((y.double() - want).abs() <= 2.0 ** -12 * want.abs() + 1e-37).all()
    assert torch.equal(q.values, ref.int8_of(want_h.float() * w)[0])
    dr, dw = torch.empty_like(h), torch.empty(cols, device="cuda")
    ws = torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(2, cols), dtype=torch.uint8, device="cuda")
    vb.vsa2_residual_norm_bwd(h, x, r, w, d_residual=dr, d_weight=dw, workspace=ws)
    grad, grad_w, size, size_w = ref.gradients(h, x, r, w, 1e-6)
    assert ((dr.double() - grad).abs() <= 2.0 ** -11 * size + 2.0 ** -8 * grad.abs()).all()
    assert ((dw.double() - grad_w).abs() <= 2.0 ** -12 * size_w + 1e-37).all()


def slices(rows):
    return [slice(0, 3), slice(rows // 2, rows // 2 + 3), slice(rows - 3, rows)]


def test_tensors_of_more_than_2_to_the_31_elements():
    """Norm, its backward, dropout and quantisation of 4.3 GB each: the first, middle and last rows as calls on these alone give them (the mask's by its definition)."""
    rows, cols = 430000, 5120
    assert rows * cols > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty(rows, cols, dtype=BF, device="cuda").normal_(generator=gen)
    h, q = torch.empty_like(x), vb.Int8.empty(rows, cols)
    f = vb.Fp8.empty(rows, cols)
    vb.vsa2_residual_norm_fwd(x, x, h=h, y_int8=q, y_fp8=f)
    for s in slices(rows):
        few_h, few_q, few_f = torch.empty(3, cols, dtype=BF, device="cuda"), vb.Int8.empty(3, cols), vb.Fp8.empty(3, cols)
        vb.vsa2_residual_norm_fwd(x[s].contiguous(), x[s].contiguous(), h=few_h, y_int8=few_q, y_fp8=few_f)
        assert torch.equal(h[s], few_h) and torch.equal(q.values[s], few_q.values) and torch.equal(q.scales[s], few_q.scales)
        assert torch.equal(f.values[s].float(), few_f.values.float()) and torch.equal(f.scales[:, s], few_f.scales)
    del f, q
    dr = torch.empty_like(x)
    vb.vsa2_residual_norm_bwd(h, x, d_residual=dr)
    for s in slices(rows):
        few = torch.empty(3, cols, dtype=BF, device="cuda")
        vb.vsa2_residual_norm_bwd(h[s].contiguous(), x[s].contiguous(), d_residual=few)
        assert torch.equal(dr[s], few)
    rng = torch.tensor([1, 2], device="cuda")
    vb.vsa2_dropout(x, dr, 0.5, rng)
    kept = ref.factors(1, 2, 3, cols, 0.5).cuda()
    assert torch.equal(dr[:3], ref.dropped(x[:3], kept).to(BF))
    last = ref.philox((torch.arange(cols // 8).numpy(), rows - 1, 2, 0), (1, 0))
    bits = torch.stack([torch.from_numpy((w >> s & 0xffff).astype("int64")) for w in last for s in (0, 16)], -1).reshape(cols).cuda()
    assert torch.equal(dr[-1] != 0, (bits >= ref.threshold(0.5)) & (x[-1] != 0))
    out = vb.Int8.empty(rows, cols)
    vb.vsa2_int8_quantize(x, out)
    for s in slices(rows):
        assert torch.equal(out.values[s], ref.int8_of(x[s].float())[0])


@pytest.mark.parametrize("m,n,k,dtype", [(150000, 15360, 64, BF), (72000, 30011, 40, F)])
def test_products_of_more_than_2_to_the_31_results(m, n, k, dtype):
    assert m * n > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(3)
    a, b = vb.Int8.empty(m, k), vb.Int8.empty(n, k)
    for v in (a, b):
        v.values.copy_(torch.randint(-128, 128, v.shape, generator=gen, device="cuda"))
        v.scales.copy_(torch.rand(v.shape[0], generator=gen, device="cuda"))
    c = torch.empty(m, n, dtype=dtype, device="cuda")
    vb.vsa2_int8_matmul(a, b, c, vb.int8_matmul_workspace(m, n, k))
    for s in slices(m):
        t = (a.values[s].double() @ b.values.double().T).float() * a.scales[s].unsqueeze(1)
        assert torch.equal(c[s], (t.double() * b.scales.double()).float().to(dtype))


def test_other_devices_and_layouts_are_refused():
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError, match="contiguous rows"):
        vb.vsa2_dropout(x.T, x.T, 0.1, torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="int64"):
        vb.vsa2_dropout(x, x, 0.1, torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="CUDA"):
        vb.vsa2_dropout(x, x, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="one shape"):
        vb.vsa2_residual_norm_fwd(x, torch.zeros(4, 65, device="cuda"), h=x)
    with pytest.raises(ValueError, match="weight"):
        vb.vsa2_residual_norm_fwd(x, weight=torch.ones(63, device="cuda"), h=x)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        vb.vsa2_residual_norm_fwd(x.half(), h=x.half())
    for bad in (lambda: vb.vsa2_residual_norm_fwd(x), lambda: vb.vsa2_residual_norm_fwd(x, h=x, p=1.0), lambda: vb.vsa2_residual_norm_fwd(x, h=x, p=0.1),
                lambda: vb.vsa2_residual_norm_fwd(x, h=x, eps=-1.0), lambda: vb.vsa2_residual_norm_fwd(x, x.bfloat16(), h=x),
                lambda: vb.vsa2_residual_norm_bwd(x, x), lambda: vb.vsa2_residual_norm_bwd(x, x, d_weight=torch.zeros(64, device="cuda")),
                lambda: vb.vsa2_dropout(x.expand(4, 64)[:1].expand(4, 64), x.clone(), 0.1, torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises(vb.Vsa2Error):
            bad()
