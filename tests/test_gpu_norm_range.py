"""Norms of rows of every size that fp32 and bf16 hold: squares of channels above 1.8e19 pass fp32's range, those of channels below 1e-23 vanish, and neither may show.

Bounds: as for the norms at ordinary sizes, 2^-19 (outputs) and 2^-18 (gradients) of the sizes that a result is made of, half a unit of bf16's last place where it is stored so; what lies below fp32's normal
numbers (2^-126) is known to its last place there, 2^-149, times the few factors it passes."""
import itertools

import pytest
import torch

from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
SIZES = [1e-44, 1e-38, 1e-30, 1e-24, 1e-20, 1e-13, 1e-7, 1.0, 1e6, 1e7, 1e12, 1e18, 2e19, 1e25, 1e32, 2e37]


def half_unit(x):
    """Half a unit of bf16's last place at x; below its normal numbers that is 2^-133 everywhere."""
    return torch.ldexp(torch.ones_like(x), (torch.frexp(x)[1] - 9).clamp(min=-134)) * (x != 0)


def problem(dim, dtype, seed=0):
    """One token a size, and among them rows of ordinary size in the same warps."""
    gen = torch.Generator(device="cuda").manual_seed(seed + dim)
    n = 2 * len(SIZES)
    x = torch.randn(1, n, 6, dim, generator=gen, device="cuda")
    size = torch.ones(n, device="cuda", dtype=torch.float64)
    size[::2] = torch.tensor(SIZES, dtype=torch.float64)
    x = (x.double() * size.view(1, n, 1, 1)).to(dtype).transpose(1, 2)
    w = [1 + 0.1 * torch.randn(dim, generator=gen, device="cuda") for _ in range(2)]
    return gen, (x[:, :3], x[:, 3:5], x[:, 5:]), w


def turned(x, inverse=False):
    """(x turned by the positions of a row of tokens, |x1| + |x2| of each channel's pair), 64 bits."""
    r = torch.arange(x.shape[2], device="cuda", dtype=torch.float64)
    angle = r[:, None] * torch.tensor([1e4 ** (-2.0 * j / x.shape[-1]) for j in range(x.shape[-1] // 2)], dtype=torch.float64, device="cuda")
    a, b = x[..., 0::2], x[..., 1::2]
    c, s = torch.cos(angle), torch.sin(angle) * (-1 if inverse else 1)
    y, size = torch.empty_like(x), torch.empty_like(x)
    y[..., 0::2], y[..., 1::2] = a * c - b * s, a * s + b * c
    size[..., 0::2] = size[..., 1::2] = a.abs() + b.abs()
    return y, size


def mean_square(x):
    return (x * x).mean(-1, keepdim=True)


@pytest.mark.parametrize("dim,dtype,out,eps", list(itertools.product((64, 128), (BF, F), (BF, F), (0.0, 1e-20, 1e-6))))
def test_forward_at_every_size(dim, dtype, out, eps):
    _, x, w = problem(dim, dtype)
    n = x[0].shape[2]
    rope = vb.vsa2_rope_plan(dim, (0, 0, dim))
    y = [torch.full((1, h, n, dim), float("nan"), dtype=out, device="cuda") for h in (3, 2, 1)]
    vb.vsa2_qkv_fwd(rope, x, y, *w, eps=eps, grid=(1, 1, n))
    eps = float(torch.tensor(eps, dtype=F))
    for i in range(2):
        xd = x[i].double()
        ms = mean_square(xd) + eps
        some = (ms > 0).expand_as(xd)                    # (with eps 0 a row of zeros has no norm)
        want, size = turned(torch.where(some, xd / ms.clamp(min=1e-300).sqrt(), 0.0) * w[i].double())
        err = (y[i].double() - want).abs()
        bound = 2.0 ** -19 * size + 2.0 ** -146 + (half_unit(want.abs() + 2.0 ** -19 * size) if out == BF else 0)
        assert ((err <= bound) | ~some).all(), [(SIZES[t // 2], float((err - bound)[:, :, t].max())) for t in range(0, n, 2)]
        assert y[i][~some].isnan().all()
    assert torch.equal(y[2], x[2].to(out))


@pytest.mark.parametrize("dim,dtype,eps", list(itertools.product((64, 128), (BF, F), (0.0, 1e-20, 1e-6))))
def test_backward_at_every_size(dim, dtype, eps):
    gen, x, w = problem(dim, dtype)
    n = x[0].shape[2]
    rope = vb.vsa2_rope_plan(dim, (0, 0, dim))
    dy = [torch.randn(1, h, n, dim, generator=gen, device="cuda") * 0.01 for h in (3, 2, 1)]
    # gradients of the size of x where 1 / x would leave fp32 (dx is about dy / x)
    ms = mean_square(x[0].double())[:, :1].sqrt()
    for d in dy:
        d.mul_(ms.clamp(min=1e-30, max=1e30).float() if eps == 0 else 1.0)
    dx = [torch.full_like(d, float("nan")) for d in dy]
    dw = [torch.empty(dim, device="cuda") for _ in range(2)]
    ws = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(dim), dtype=torch.uint8, device="cuda")
    vb.vsa2_qkv_bwd(rope, x, dy, dx, *w, *dw, ws, eps=eps, grid=(1, 1, n))
    eps = float(torch.tensor(eps, dtype=F))
    for i in range(2):
        xd, wd = x[i].double(), w[i].double()
        ms = mean_square(xd) + eps
        some = (ms > 0).expand_as(xd)
        r = torch.where(ms > 0, ms.clamp(min=1e-300).rsqrt(), 0.0)
        g, size = turned(dy[i].double(), inverse=True)
        hat, wg = xd * r, g * wd
        want = r * (wg - hat * (wg * hat).mean(-1, keepdim=True))
        size = r * (size * wd.abs() + hat.abs() * (size * wd.abs() * hat.abs()).mean(-1, keepdim=True))
        err = (dx[i].double() - want).abs()
        # (g itself may lie below the normal numbers: its last place, 2^-149, times r)
        bound = 2.0 ** -18 * size + 2.0 ** -146 * (1 + r)
        fits = some & (want.abs() < 3e38)
        assert ((err <= bound) | ~fits).all(), [(SIZES[t // 2], float((err - bound)[:, :, t].max())) for t in range(0, n, 2)]
        if some.all():
            terms = g * hat
            assert ((dw[i].double() - terms.sum((0, 1, 2))).abs() <= 2.0 ** -14 * terms.abs().sum((0, 1, 2)) + 1e-38).all()


@pytest.mark.parametrize("layout", [vb.ROPE_PAIRS, vb.ROPE_HALVES])
def test_ordinary_rows_do_not_depend_on_their_neighbours_sizes(layout):
    gen = torch.Generator(device="cuda").manual_seed(5)
    rope, n = vb.vsa2_rope_plan(64, (16, 16, 32), layout=layout), 24
    x = torch.randn(1, 5, n, 64, generator=gen, device="cuda")
    w = [1 + 0.1 * torch.randn(64, generator=gen, device="cuda") for _ in range(2)]
    dy = torch.randn(1, 5, n, 64, generator=gen, device="cuda")
    odd = x.clone()
    odd[:, ::2, 1::3] *= 1e25
    odd[:, 1::2, 2::3] *= 1e-30
    same = (odd == x).all(-1)
    got = []
    for v in (x, odd):
        y, dx = [torch.empty(1, 5, n, 64, device="cuda") for _ in range(3)], [torch.empty(1, 5, n, 64, device="cuda") for _ in range(3)]
        vb.vsa2_qkv_fwd(rope, (v,) * 3, y, *w, eps=1e-12, grid=(2, 3, 4))
        ws = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(64), dtype=torch.uint8, device="cuda")
        vb.vsa2_qkv_bwd(rope, (v,) * 3, (dy,) * 3, dx, *w, None, None, ws, eps=1e-12, grid=(2, 3, 4))
        got.append((*y[:2], *dx[:2]))
    assert all(torch.equal(a[same], b[same]) for a, b in zip(*got))
    assert same.any() and not same.all() and all(t.isfinite().all() for t in got[1])
