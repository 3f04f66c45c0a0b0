"""GPU parity of the norm of the residual stream, forward and backward, against its formulas in 64 bits."""
import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
# What fp32 arithmetic leaves of a normed row: a sum of squares is added up in at most 40 steps one behind the other (8 a piece, 4 pieces, 5 + 4 across threads; positive terms, 2^-24
# each) and its root halves that; the reciprocal root is 2 ulp off, the products four more roundings: 20 + 4 + 4 < 2^5 of 2^-24.  Rows of more than 8192 elements add 8 steps for each
# 8192; those here have 40,000, 8 x 5 more.  Twice that, 2^-18.
FINE = 2.0 ** -18


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def make(rows, cols, dtype, gen, size=1.0):
    return (torch.randn(rows, cols, generator=gen, device="cuda") * size).to(dtype)


def rng_of(seed, offset):
    wrap = lambda v: (v + 2 ** 63) % 2 ** 64 - 2 ** 63
    return torch.tensor([wrap(seed), wrap(offset)], device="cuda")


def check_forward(x, residual, w, eps, p, seed, offset, f32_out=True, pad=0):
    """Every output at once, each against its definition."""
    rows, cols = x.shape
    factor = ref.factors(seed, offset, rows, cols, p) if p else None
    want_h = ref.stream(x, residual, factor)
    room = torch.full((rows, cols + pad), 7.0, dtype=want_h.dtype, device="cuda")
    h, y = room[:, :cols], torch.full((rows, cols), float("nan"), dtype=F if f32_out else BF, device="cuda")
    y_fp8, y_int8 = vb.Fp8.empty(rows, cols), vb.Int8.empty(rows, cols)
    y_fp8.scales.fill_(77)
    vb.vsa2_residual_norm_fwd(x, residual, w, eps=eps, h=h, y=y, y_fp8=y_fp8, y_int8=y_int8, p=p, rng=rng_of(seed, offset) if p else None)
    assert torch.equal(h, want_h)
    assert (room[:, cols:] == 7.0).all()
    want, r = ref.normed(want_h, w, eps)
    off = (y.double() - want).abs()
    assert (off <= (FINE + half_step(y.dtype)) * want.abs() + 1e-37).all(), float((off / want.abs().clamp(min=1e-30)).max())
    # e4m3: the scale is the least power of two that holds the block's largest, which fp32 may see a little differently
    e = y_fp8.scales.transpose(0, 1).reshape(rows, -1)
    blocks = -(-cols // 128)
    assert not e[:, blocks:].any()
    scale = torch.exp2(e[:, :blocks].double() - 127)
    top = torch.nn.functional.pad(want.abs(), (0, blocks * 128 - cols)).view(rows, blocks, 128).amax(dim=2)
    assert (top <= 448 * scale * (1 + FINE)).all() and ((top >= 224 * scale * (1 - FINE)) | (e[:, :blocks] == 0)).all()
    each = scale.repeat_interleave(128, dim=1)[:, :cols]
    off = (y_fp8.values.float().double() * each - want).abs()
    assert (off <= (FINE + 2.0 ** -4) * want.abs() + each * 2.0 ** -10).all()
    # int8: values exactly, the scale as the norm's factor allows
    v = want_h.float() if w is None else want_h.float() * w
    q, m, fine = ref.int8_of(v)
    assert fine.all() and torch.equal(y_int8.values, q)
    want_scale = m.double() / 127 * r.squeeze(1)
    assert ((y_int8.scales.double() - want_scale).abs() <= FINE * want_scale + 1e-44).all()


SIZES = [(1, 1), (1, 5120), (3, 7), (2, 8), (5, 64), (33, 129), (64, 513), (7, 1000), (130, 1536), (1, 4096), (9, 4104), (300, 2048), (17, 5120), (3, 8200), (2, 16384), (3, 16392), (2, 40003)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("x_type,stream_type", [(BF, BF), (BF, F), (F, F), (F, BF)])
def test_forward(rows, cols, x_type, stream_type):
    gen = torch.Generator(device="cuda").manual_seed(rows * 31 + cols)
    x, r = make(rows, cols, x_type, gen), make(rows, cols, stream_type, gen, 2.0)
    w = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
    check_forward(x, r, w, 1e-6, 0.0, 0, 0, f32_out=rows % 2 == 1)
    check_forward(x, None, None, 1e-5, 0.3, 5, 2 ** 40 + 3, f32_out=rows % 2 == 0)


@pytest.mark.parametrize("cols,pad,skip", [(1536, 8, 0), (1536, 3, 0), (1530, 0, 0), (1536, 8, 3), (600, 11, 1), (9001, 0, 0), (20011, 2, 1)])
def test_rows_of_any_stride_and_address(cols, pad, skip):
    gen = torch.Generator(device="cuda").manual_seed(cols + pad)
    w = (1 + 0.1 * torch.randn(cols + 3, generator=gen, device="cuda"))[skip:skip + cols]
    x, r = make(9, cols + pad + skip, BF, gen)[:, skip:skip + cols], make(9, cols + pad + skip, F, gen)[:, skip:skip + cols]
    check_forward(x, r, w, 1e-6, 0.25, 2 ** 33 + 1, 4, pad=pad)
    check_forward(r, x, w, 1e-6, 0.0, 0, 0, pad=pad)


def test_in_place_and_each_output_alone():
    gen = torch.Generator(device="cuda").manual_seed(1)
    for cols in (1536, 20000):
        x, r, w = make(40, cols, BF, gen), make(40, cols, BF, gen), 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
        h, y, f, q = torch.empty_like(r), torch.empty_like(x), vb.Fp8.empty(40, cols), vb.Int8.empty(40, cols)
        rng = rng_of(3, 4)
        vb.vsa2_residual_norm_fwd(x, r, w, h=h, y=y, y_fp8=f, y_int8=q, p=0.1, rng=rng)
        stream, out = r.clone(), x.clone()
        vb.vsa2_residual_norm_fwd(out, stream, w, h=stream, y=out, p=0.1, rng=rng)      # the stream's own memory, and the branch's
        assert torch.equal(stream, h) and torch.equal(out, y)
        f2, q2, y2, h2 = vb.Fp8.empty(40, cols), vb.Int8.empty(40, cols), torch.empty_like(y), torch.empty_like(h)
        for outs in ({"y_fp8": f2}, {"y_int8": q2}, {"y": y2}, {"h": h2}):
            vb.vsa2_residual_norm_fwd(x, r, w, p=0.1, rng=rng, **outs)
        assert torch.equal(f2.values.float(), f.values.float()) and torch.equal(f2.scales, f.scales)
        assert torch.equal(q2.values, q.values) and torch.equal(q2.scales, q.scales) and torch.equal(y2, y) and torch.equal(h2, h)


@pytest.mark.parametrize("cols", [1536, 20000])
def test_rows_of_any_finite_size(cols):
    gen = torch.Generator(device="cuda").manual_seed(2)
    sizes = torch.tensor([1e-38, 1e-30, 1e-20, 1e-12, 1.0, 1e12, 1e19, 1e30, 1e37, 0.0], device="cuda").unsqueeze(1)
    x = torch.randn(10, cols, generator=gen, device="cuda").clamp(-3, 3) * sizes
    w = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
    y, q = torch.empty_like(x), vb.Int8.empty(10, cols)
    for eps in (0.0, 1e-6):
        vb.vsa2_residual_norm_fwd(x, weight=w, eps=eps, y=y, y_int8=q)
        want, r = ref.normed(x, w, eps)
        some = slice(0, 9 if eps == 0 else 10)
        # (the smallest row holds subnormal numbers: their products with a power of two are exact, so nothing is lost)
        assert ((y.double() - want).abs()[some] <= FINE * want.abs()[some] + 1e-37).all()
        assert y[9].isnan().all() if eps == 0 else (y[9] == 0).all()
        # (an element of a scaled row may round to the neighbouring whole number where its product is half way)
        deq = q.values.double() * q.scales.double().unsqueeze(1)
        top = want.abs().amax(dim=1, keepdim=True)
        # (the scale is that of max |h w|, or of 2^-100 where the largest is smaller, times the norm's factor: with eps the first row's step is 1000 * 2^-100 / 127, above its values)
        step = torch.maximum(top, 2.0 ** -100 * r if eps else 0 * top) / 127
        assert ((deq - want).abs()[some] <= step[some] * (0.5 + 2.0 ** -12) + 1e-37).all()
        d = torch.randn(10, cols, generator=gen, device="cuda")
        dr = torch.empty_like(x)
        vb.vsa2_residual_norm_bwd(x, d, weight=w, eps=eps, d_residual=dr)
        rows = slice(1 if eps == 0 else 0, 9)      # (1 / |h| of the first row without eps is beyond fp32)
        grad, _, size, _ = ref.gradients(x[rows], d[rows], None, w, eps)
        assert ((dr[rows].double() - grad).abs() <= 2 * FINE * size + 1e-37).all()


def test_what_is_not_finite_stays_in_its_row():
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, w = make(6, 700, F, gen), 1 + 0.1 * torch.randn(700, generator=gen, device="cuda")
    clean = x.clone()
    x[1, 5], x[3, 699], x[4, 0], x[4, 300] = float("inf"), float("nan"), float("-inf"), float("inf")
    y, f, q = torch.empty_like(x), vb.Fp8.empty(6, 700), vb.Int8.empty(6, 700)
    vb.vsa2_residual_norm_fwd(x, weight=w, y=y, y_fp8=f, y_int8=q)
    want = ref.normed(clean, w, 1e-6)[0]
    for row in (0, 2, 5):
        assert ((y[row].double() - want[row]).abs() <= FINE * want[row].abs()).all() and q.scales[row].isfinite()
    assert y[1, 5].isnan() and (y[1, 6:] == 0).all() and y[3].isnan().all() and y[4, 0].isnan()
    assert q.scales[[1, 3, 4]].isnan().all() and not q.values[[1, 3, 4]].any()
    assert f.values[1].float()[5].isnan() and f.values[3].float().isnan().all() and (f.values[1].float()[6:] == 0).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 5120), (3, 7), (33, 129), (700, 64), (130, 1536), (2500, 1536), (40, 1000), (1300, 5120), (3, 8192), (5, 8200), (1190, 8201), (3, 40003)])
@pytest.mark.parametrize("stream_type,dy_type", [(BF, BF), (F, BF), (F, F), (BF, F)])
def test_backward(rows, cols, stream_type, dy_type):
    gen = torch.Generator(device="cuda").manual_seed(rows * 3 + cols)
    h, dy, dh = make(rows, cols, stream_type, gen, 2.0), make(rows, cols, dy_type, gen), make(rows, cols, stream_type, gen)
    w = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
    ws = torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    p, dx_type = (0.2, BF) if rows % 2 else (0.0, F)
    dr, dx, dw = torch.empty_like(h), torch.empty(rows, cols, dtype=dx_type, device="cuda"), torch.full((cols,), float("nan"), device="cuda")
    vb.vsa2_residual_norm_bwd(h, dy, dh, w, d_residual=dr, dx=dx, d_weight=dw, workspace=ws, p=p, rng=rng_of(9, 8))
    grad, grad_w, size, size_w = ref.gradients(h, dy, dh, w, 1e-6)
    # two sums of fp32 products, of which the second's terms have signs: its error goes with the sum of their magnitudes
    assert ((dr.double() - grad).abs() <= 2 * FINE * size + half_step(stream_type) * grad.abs()).all()
    factor = ref.factors(9, 8, rows, cols, p).cuda()
    assert ((dx.double() - grad * factor).abs() <= (2 * FINE * size + half_step(dx_type) * grad.abs()) * factor + 2.0 ** -24 * (grad * factor).abs()).all()
    # a column's terms: one behind the other in a CTA (3 at most of 148 CTAs at these sizes .. 17), then 1184 / 8 parts and 8: 2^8 of 2^-24, and the normed row's own error
    assert ((dw.double() - grad_w).abs() <= (FINE + 2.0 ** -16) * size_w + 1e-37).all()
    # each output alone, without a gradient from the stream, and again: the same bits
    for outs in ({"d_residual": dr}, {"dx": dx}, {"d_weight": dw, "workspace": ws}):
        name = next(iter(outs))
        before = outs[name].clone()
        outs[name].fill_(float("nan"))
        vb.vsa2_residual_norm_bwd(h, dy, dh, w, p=p, rng=rng_of(9, 8), **outs)
        assert torch.equal(outs[name], before), name
    vb.vsa2_residual_norm_bwd(h, dy, None, None, d_residual=dr)
    grad, _, size, _ = ref.gradients(h, dy, None, None, 1e-6)
    assert ((dr.double() - grad).abs() <= 2 * FINE * size + half_step(stream_type) * grad.abs()).all()


def test_backward_of_strided_rows_and_in_place():
    gen = torch.Generator(device="cuda").manual_seed(5)
    for cols, pad in ((1530, 3), (1536, 8), (9001, 5)):
        h, dy, dh = (make(50, cols + pad, BF, gen)[:, pad:] for _ in range(3))
        grad, _, size, _ = ref.gradients(h, dy, dh, None, 1e-6)
        stream = dh.clone() if pad == 8 else dh
        vb.vsa2_residual_norm_bwd(h, dy, stream, d_residual=stream)      # written over the gradient that arrives
        assert ((stream.double() - grad).abs() <= 2 * FINE * size + half_step(BF) * grad.abs()).all()


def test_gradients_against_differences():
    """Central differences of the forward kernel along random directions: their own error is seen in halving the step, and fp32 leaves FINE of the terms over the step."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    rows, cols, p = 4, 96, 0.25
    x, r, c, d = (make(rows, cols, F, gen) for _ in range(4))
    w, dw_dir = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    rng = rng_of(11, 12)
    h, y = torch.empty_like(x), torch.empty_like(x)

    def loss(x, r, w):
        vb.vsa2_residual_norm_fwd(x, r, w, h=h, y=y, p=p, rng=rng)
        return float((y.double() * c.double()).sum()), float((y.double() * c.double()).abs().sum())

    loss(x, r, w)
    dr, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    vb.vsa2_residual_norm_bwd(h.clone(), c, None, w, d_residual=dr, dx=dx, d_weight=dw, workspace=ws, p=p, rng=rng)
    for grad, direction, at in ((dx, d, lambda t: (x + t * d, r, w)), (dr, d, lambda t: (x, r + t * d, w)), (dw, dw_dir, lambda t: (x, r, w + t * dw_dir))):
        got = float((grad.double() * direction.double()).sum())
        step = 2.0 ** -5
        halves = [(loss(*at(s))[0] - loss(*at(-s))[0]) / (2 * s) for s in (step, step / 2)]
        noise = 4 * FINE * loss(x, r, w)[1] / step
        assert abs(got - halves[1]) <= abs(halves[0] - halves[1]) + noise, (got, halves, noise)


def test_sizes_of_zero():
    for rows, cols in ((0, 64), (5, 0), (0, 0)):
        x = torch.empty(rows, cols, device="cuda")
        vb.vsa2_residual_norm_fwd(x, h=torch.empty_like(x), y_int8=vb.Int8.empty(rows, cols), y_fp8=vb.Fp8.empty(rows, cols))
        dw = torch.full((cols,), 5.0, device="cuda")
        ws = torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        vb.vsa2_residual_norm_bwd(x, x, d_residual=torch.empty_like(x), d_weight=dw, workspace=ws)
        assert (dw == 0).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("cols", [1, 7, 9, 250, 255, 511, 1024, 2041, 2047, 2049, 4100, 8191, 8200, 9000])
def test_rows_at_every_address(dtype, cols):
    """Matrices of one odd stride whose rows begin at every offset from a 16-byte boundary; what lies around the rows stays, also in place."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rows, ld = 17, cols + 5 + cols % 2
    rooms = [make(rows + 1, ld, dtype, gen) for _ in range(3)]
    view = lambda room, skip: torch.as_strided(room, (rows, cols), (ld, 1), skip)
    for skip in (0, 1, 3):
        x, r = view(rooms[0], skip), view(rooms[1], (skip + 2) % 5)
        out = torch.full_like(rooms[2], 7.0)
        y = view(out, (skip + 1) % 4)
        keep = out.clone()
        h = torch.empty(rows, cols, dtype=dtype, device="cuda")
        vb.vsa2_residual_norm_fwd(x, r, None, h=h, y=y, p=0.25, rng=rng_of(skip, 1))
        want_h = ref.stream(x, r, ref.factors(skip, 1, rows, cols, 0.25))
        assert torch.equal(h, want_h)
        want, _ = ref.normed(want_h, None, 1e-6)
        assert ((y.double() - want).abs() <= (FINE + half_step(dtype)) * want.abs() + 1e-37).all()
        y.copy_(view(keep, (skip + 1) % 4))
        assert torch.equal(out, keep)                             # nothing else was written
        again = rooms[1].clone()
        stream = view(again, (skip + 2) % 5)
        vb.vsa2_residual_norm_fwd(x, stream, None, h=stream, p=0.25, rng=rng_of(skip, 1))
        assert torch.equal(stream, want_h)
        stream.copy_(r)
        assert torch.equal(again, rooms[1])
        dr = view(out, (skip + 1) % 4)
        vb.vsa2_residual_norm_bwd(h, x, r, d_residual=dr)
        grad, _, size, _ = ref.gradients(h, x, r, None, 1e-6)
        assert ((dr.double() - grad).abs() <= 2 * FINE * size + half_step(dtype) * grad.abs() + 1e-37).all()
        dr.copy_(view(keep, (skip + 1) % 4))
        assert torch.equal(out, keep)
        d = view(out, (skip + 3) % 6)
        vb.vsa2_dropout(x, d, 0.5, rng_of(skip, 2), residual=r)
        assert torch.equal(d, (r.float() + ref.dropped(x, ref.factors(skip, 2, rows, cols, 0.5))).to(dtype))
        d.copy_(view(keep, (skip + 3) % 6))
        assert torch.equal(out, keep)
        q = vb.Int8.empty(rows, cols)
        vb.vsa2_int8_quantize(x, q)
        assert torch.equal(q.values, ref.int8_of(x.float())[0])
