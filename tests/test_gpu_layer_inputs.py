"""GPU parity of rotary positions, and of the norms of q and k with the rotation in the same pass, against their definitions in 64 bits.

Bounds (derived): an angle is 2^-32 turns off at most, a sine or cosine then 2^-22; a rotated channel is a sum of two products, so fp32 results lie
within 2^-20 of |x1| + |x2|.  A norm adds a sum of D squares and a reciprocal root, together below 2^-20 relative.  What is stored in bf16 adds half
a unit of its last place."""
import itertools
import math

import numpy as np
import pytest
import torch

from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def angles(channels, grid, first, n, positions=None, theta=(1e4,) * 3, scale=(1.0,) * 3):
    """Angle of every pair at every token, 64 bits, [batch or 1, n, pairs]."""
    if positions is None:
        t, h, w = grid
        r = torch.arange(first, first + n, device="cuda")
        pos = torch.stack([r // (h * w), r // w % h, r % w], dim=-1) * (r < t * h * w).unsqueeze(-1)
    else:
        pos = positions
    pos = pos.reshape(-1, n, 3).double()
    parts = [scale[a] * pos[..., a:a + 1] * torch.tensor([theta[a] ** (-2.0 * j / c) for j in range(c // 2)], dtype=torch.float64, device="cuda")
             for a, c in enumerate(channels)]
    return torch.cat(parts, dim=-1).unsqueeze(1)


def halves_of(x, pairs, layout):
    if layout == vb.ROPE_HALVES:
        return x[..., :pairs], x[..., pairs:2 * pairs]
    return x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]


def joined(a, b, x, pairs, layout):
    y = x.clone()
    halves_of(y, pairs, layout)[0].copy_(a)
    halves_of(y, pairs, layout)[1].copy_(b)
    return y


def turned(x, angle, layout, inverse=False):
    """(turned x, |x1| + |x2| of each channel's pair), 64 bits."""
    pairs = angle.shape[-1]
    a, b = halves_of(x, pairs, layout)
    c, s = torch.cos(angle), torch.sin(angle) * (-1.0 if inverse else 1.0)
    size = a.abs() + b.abs()
    return joined(a * c - b * s, a * s + b * c, x, pairs, layout), joined(size, size, x.abs(), pairs, layout)


def half_unit(x):
    """Half a unit of bf16's last place (8 significant bits) at x: 2^(e - 8) for 2^e <= |x| < 2^(e + 1)."""
    return torch.ldexp(torch.ones_like(x), torch.frexp(x)[1] - 9) * (x != 0)


def close(got, want, size, relative=2.0 ** -20):
    assert got.shape == want.shape
    err = (got.double() - want).abs()
    bound = relative * size + 1e-38 + (half_unit(want.abs() + relative * size) if got.dtype == BF else 0)
    bad = ~(err <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} out of bounds, worst {float((err - bound).max()):.3g}"


def randn(gen, *shape, dtype=BF, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


ROPES = [(64, (16, 24, 24), vb.ROPE_PAIRS), (64, (0, 32, 32), vb.ROPE_HALVES), (64, (2, 0, 6), vb.ROPE_PAIRS), (64, (16, 0, 0), vb.ROPE_HALVES),
         (128, (44, 42, 42), vb.ROPE_PAIRS), (128, (44, 42, 42), vb.ROPE_HALVES), (128, (0, 0, 128), vb.ROPE_HALVES), (128, (0, 0, 0), vb.ROPE_PAIRS)]


@pytest.mark.parametrize("dim,channels,layout", ROPES)
@pytest.mark.parametrize("grid,text,first,heads,batch,tin,tout", [
    ((1, 1, 1), 0, 0, 1, 1, BF, BF),               # one token
    ((3, 5, 7), 9, 0, 3, 2, F, F),                 # text rows behind the grid
    ((2, 3, 11), 5, 17, 5, 1, BF, F),              # a part of the rows
    ((2, 5, 13), 0, 0, 2, 3, F, BF),
])
def test_rotation_and_its_inverse(dim, channels, layout, grid, text, first, heads, batch, tin, tout):
    gen = torch.Generator(device="cuda").manual_seed(dim + first)
    n = grid[0] * grid[1] * grid[2] + text - first
    theta, scale = (1e4, 500.0, 1e6), (1.0, 0.5, 2.0)
    rope = vb.vsa2_rope_plan(dim, channels, theta=theta, scale=scale, layout=layout)
    x = randn(gen, batch, heads, n, dim, dtype=tin)
    angle = angles(channels, grid, first, n, theta=theta, scale=scale)
    for inverse in (False, True):
        y = torch.full((batch, heads, n, dim), float("nan"), dtype=tout, device="cuda")
        vb.vsa2_rope_apply(rope, x, y, grid=grid, first=first, inverse=inverse)
        close(y, *turned(x.double(), angle, layout, inverse))
        rest = 2 * angle.shape[-1]
        assert torch.equal(y[..., rest:], x[..., rest:].to(tout))          # channels that do not turn
        if text and first == 0:
            assert torch.equal(y[:, :, n - text:], x[:, :, n - text:].to(tout))


@pytest.mark.parametrize("layout", [vb.ROPE_PAIRS, vb.ROPE_HALVES])
def test_positions_from_a_list_of_any_size(layout):
    """Negative positions, and positions where position * frequency in fp32 would be radians off."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, channels = 37, (16, 24, 24)
    rope = vb.vsa2_rope_plan(64, channels, layout=layout)
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, n, 3), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    pos[:, 0] = torch.tensor([-1, 0, 1])
    pos[:, 1] = torch.tensor([2 ** 31 - 1, -2 ** 31, 65537])
    x = randn(gen, 2, 3, n, 64, dtype=F)
    y = torch.empty_like(x)
    # the frequencies' own rounding in 64 bits is 2^-53 * 2^31 turns at these positions: below the bound
    for p in (pos, pos[:1].contiguous(), pos[0].contiguous()):
        vb.vsa2_rope_apply(rope, x, y, positions=p)
        want, size = turned(x.double(), angles(channels, None, 0, n, positions=p), layout)
        close(y, want, size)


def test_large_positions_and_rows_beyond_32_bits_of_offset():
    """A view whose rows lie 2^31 elements and more apart (a slice of a long buffer)."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    apart = 2 ** 31 + 64
    room = torch.empty(apart + 2 * 64, dtype=BF, device="cuda")
    x = room.as_strided((1, 2, 2, 64), (64, apart, 64, 1))
    x.copy_(randn(gen, 1, 2, 2, 64))
    rope = vb.vsa2_rope_plan(64, (0, 0, 64))
    y = torch.empty(1, 2, 2, 64, dtype=BF, device="cuda")
    vb.vsa2_rope_apply(rope, x, y, grid=(1, 1, 2))
    close(y, *turned(x.double(), angles((0, 0, 64), (1, 1, 2), 0, 2), vb.ROPE_PAIRS))


@pytest.mark.parametrize("layout", [vb.ROPE_PAIRS, vb.ROPE_HALVES])
def test_in_place_strided_and_broadcast_views(layout):
    gen = torch.Generator(device="cuda").manual_seed(5)
    rope = vb.vsa2_rope_plan(128, (32, 32, 32), layout=layout)
    grid, n = (3, 4, 9), 108
    angle = angles((32, 32, 32), grid, 0, n)
    packed = randn(gen, 2, n, 7, 128)
    x = packed.transpose(1, 2)[:, 2:5]                                     # token-major, some of the heads
    want, size = turned(x.double(), angle, layout)
    rest = packed.clone()
    vb.vsa2_rope_apply(rope, x, x, grid=grid)                              # in place
    close(x, want, size)
    assert torch.equal(packed[:, :, :2], rest[:, :, :2]) and torch.equal(packed[:, :, 5:], rest[:, :, 5:])
    one = randn(gen, 1, 1, n, 128).expand(2, 3, n, 128)                    # one head for all
    y = torch.empty(2, n, 3, 128, dtype=BF, device="cuda").transpose(1, 2)
    vb.vsa2_rope_apply(rope, one, y, grid=grid)
    close(y, *turned(one.double(), angle, layout))


def test_rotation_keeps_lengths_and_undoes_itself():
    gen = torch.Generator(device="cuda").manual_seed(6)
    rope = vb.vsa2_rope_plan(128, (44, 42, 42))
    x = randn(gen, 1, 4, 21 * 9 * 16, 128, dtype=F)
    y, z = torch.empty_like(x), torch.empty_like(x)
    vb.vsa2_rope_apply(rope, x, y, grid=(21, 9, 16))
    vb.vsa2_rope_apply(rope, y, z, grid=(21, 9, 16), inverse=True)
    assert float((z - x).abs().max()) <= 2.0 ** -18 * float(x.abs().max())
    assert float((y.norm(dim=-1) / x.norm(dim=-1) - 1).abs().max()) <= 2.0 ** -18


# ------------------------------------------------------------------------------------------------------------- norms, rotation, heads
class Problem:
    def __init__(self, batch, hq, hk, grid, text, dim, channels, layout, *, first=0, x_dtype=BF, g_dtype=BF, seed=0, norm=True, eps=1e-6,
                 size=1.0, turn=True):
        gen = torch.Generator(device="cuda").manual_seed(seed + hq)
        self.n = n = grid[0] * grid[1] * grid[2] + text - first
        self.rope = vb.vsa2_rope_plan(dim, channels, layout=layout) if turn else None
        self.layout, self.dim, self.heads = layout, dim, (hq, hk, hk)
        self.kw = dict(grid=grid, first=first, norm=norm, eps=eps)
        self.norm, self.eps = norm, eps
        self.angle = angles(channels if turn else (0, 0, 0), grid, first, n)
        self.packed = randn(gen, batch, n, hq + 2 * hk, dim, dtype=x_dtype, scale=size)
        v = self.packed.transpose(1, 2)
        self.x = (v[:, :hq], v[:, hq:hq + hk], v[:, hq + hk:])
        self.w = [1.0 + 0.2 * randn(gen, dim, dtype=F) for _ in range(2)]
        self.dy = [randn(gen, batch, h, n, dim, dtype=g_dtype) for h in self.heads]
        self.gen, self.batch = gen, batch

    def forward(self, dtype=BF):
        y = [torch.full((self.batch, h, self.n, self.dim), float("nan"), dtype=dtype, device="cuda") for h in self.heads]
        vb.vsa2_qkv_fwd(self.rope, self.x, y, *self.w, **self.kw)
        return y

    def hat(self, i):
        x = self.x[i].double()
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.eps) if self.norm else x

    def check_forward(self, y):
        for i in range(2):
            x = self.hat(i) * self.w[i].double() if self.norm else self.hat(i)
            close(y[i], *turned(x, self.angle, self.layout), relative=2.0 ** -19)
        assert torch.equal(y[2], self.x[2].to(y[2].dtype))

    def backward(self, dtype=BF):
        dx = torch.full((self.batch, self.n, sum(self.heads), self.dim), float("nan"), dtype=dtype, device="cuda")
        v, (hq, hk, _) = dx.transpose(1, 2), self.heads
        dw = [torch.full((self.dim,), float("nan"), device="cuda") for _ in range(2)]
        ws = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(self.dim), dtype=torch.uint8, device="cuda")
        vb.vsa2_qkv_bwd(self.rope, self.x, self.dy, (v[:, :hq], v[:, hq:hq + hk], v[:, hq + hk:]), *self.w, *dw, ws, **self.kw)
        return (v[:, :hq], v[:, hq:hq + hk], v[:, hq + hk:]), dw

    def check_backward(self, dx, dw):
        for i in range(2):
            g, size = turned(self.dy[i].double(), self.angle, self.layout, inverse=True)
            if not self.norm:
                close(dx[i], g, size)
                assert not dw[i].any()
                continue
            x, w = self.x[i].double(), self.w[i].double()
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + self.eps)
            hat, wg = x * r, g * w
            want = r * (wg - hat * (wg * hat).mean(-1, keepdim=True))
            size = r * (size * w.abs() + hat.abs() * (size * w.abs() * hat.abs()).mean(-1, keepdim=True))
            close(dx[i], want, size, relative=2.0 ** -18)
            terms = g * hat
            # sums of up to 2^10 terms in a row, then of the parts
            assert ((dw[i].double() - terms.sum((0, 1, 2))).abs() <= 2.0 ** -14 * terms.abs().sum((0, 1, 2)) + 1e-30).all()
        assert torch.equal(dx[2], self.dy[2].to(dx[2].dtype))


QKV = [
    dict(batch=1, hq=1, hk=1, grid=(1, 1, 1), text=0, dim=64, channels=(16, 24, 24), layout=vb.ROPE_PAIRS),               # one token
    dict(batch=2, hq=4, hk=2, grid=(3, 5, 7), text=3, dim=64, channels=(0, 32, 32), layout=vb.ROPE_HALVES),
    dict(batch=1, hq=6, hk=6, grid=(2, 9, 5), text=0, dim=128, channels=(44, 42, 42), layout=vb.ROPE_PAIRS),
    dict(batch=3, hq=5, hk=1, grid=(2, 3, 11), text=18, dim=128, channels=(16, 56, 56), layout=vb.ROPE_HALVES, first=13),
    dict(batch=1, hq=12, hk=3, grid=(5, 14, 23), text=77, dim=128, channels=(44, 42, 42), layout=vb.ROPE_PAIRS, x_dtype=F, g_dtype=F),
    dict(batch=2, hq=40, hk=40, grid=(1, 2, 3), text=0, dim=64, channels=(16, 24, 24), layout=vb.ROPE_PAIRS),             # many heads, few tokens
    dict(batch=1, hq=2, hk=1, grid=(4, 31, 33), text=0, dim=128, channels=(32, 32, 32), layout=vb.ROPE_PAIRS, norm=False),
    dict(batch=1, hq=3, hk=3, grid=(2, 3, 4), text=0, dim=128, channels=(0, 0, 0), layout=vb.ROPE_PAIRS, turn=False, g_dtype=F),
    dict(batch=1, hq=2, hk=2, grid=(2, 3, 4), text=0, dim=64, channels=(16, 24, 24), layout=vb.ROPE_PAIRS, size=1e-4),    # eps matters
    dict(batch=1, hq=2, hk=2, grid=(2, 3, 4), text=0, dim=64, channels=(16, 24, 24), layout=vb.ROPE_PAIRS, size=1e4),
]


@pytest.mark.parametrize("i,dtype", list(itertools.product(range(len(QKV)), (BF, F))))
def test_norms_rotation_and_heads_forward(i, dtype):
    p = Problem(seed=i, **QKV[i])
    p.check_forward(p.forward(dtype))


@pytest.mark.parametrize("i,dtype", list(itertools.product(range(len(QKV)), (BF, F))))
def test_norms_rotation_and_heads_backward(i, dtype):
    p = Problem(seed=100 + i, **QKV[i])
    dx, dw = p.backward(dtype)
    p.check_backward(dx, dw)
    again, dw2 = p.backward(dtype)
    assert all(torch.equal(a, b) for a, b in zip((*dx, *dw), (*again, *dw2)))       # sums run in a fixed order


@pytest.mark.parametrize("layout", [vb.ROPE_PAIRS, vb.ROPE_HALVES])
def test_gradients_against_differences(layout):
    """Directional derivatives of sum(y * c) by central differences of the forward in fp32: the difference quotient's own error is eps^2
    of the third derivative plus rounding, both below 2e-3 at this step."""
    p = Problem(1, 2, 1, (2, 3, 4), 3, 64, (16, 24, 24) if layout == vb.ROPE_PAIRS else (16, 16, 32), layout, x_dtype=F, g_dtype=F, seed=8)
    dx, dw = p.backward(F)
    step = 2.0 ** -7

    def value():
        return sum(float((y.double() * c.double()).sum()) for y, c in zip(p.forward(F), p.dy))

    for i in range(3):
        d = torch.sign(randn(p.gen, *p.x[i].shape, dtype=F))
        keep, grad = p.packed.clone(), float((dx[i].double() * d.double()).sum())
        p.x[i].add_(d, alpha=step)
        up = value()
        p.packed.copy_(keep)
        p.x[i].sub_(d, alpha=step)
        down = value()
        p.packed.copy_(keep)
        scale = float((dx[i].double() ** 2).sum().sqrt()) * math.sqrt(d.numel()) / math.sqrt(p.n)
        assert abs((up - down) / (2 * step) - grad) <= 5e-3 * scale
    for i in range(2):
        d = torch.sign(randn(p.gen, p.dim, dtype=F))
        keep, grad = p.w[i].clone(), float((dw[i].double() * d.double()).sum())
        p.w[i] = keep + step * d
        up = value()
        p.w[i] = keep - step * d
        down = value()
        p.w[i] = keep
        assert abs((up - down) / (2 * step) - grad) <= 1e-3 * float(dw[i].double().norm()) * math.sqrt(p.dim)


def test_rows_of_zeros_infinities_and_nan_stay_in_their_rows():
    p = Problem(1, 2, 2, (2, 3, 4), 0, 64, (16, 24, 24), vb.ROPE_PAIRS, seed=9)
    clean = p.forward()
    p.packed[0, 3, 0] = 0
    p.packed[0, 4, 1, 5] = float("inf")
    p.packed[0, 5, 2, 7] = float("nan")
    y = p.forward()
    assert not y[0][0, 0, 3].any()                                                   # zeros over sqrt(eps)
    assert y[0][0, 1, 4].isnan().any() and y[1][0, 0, 5].isnan().all()
    y[0][0, 0, 3], y[0][0, 1, 4], y[1][0, 0, 5] = (clean[0][0, 0, 3], clean[0][0, 1, 4], clean[1][0, 0, 5])
    assert all(torch.equal(a, b) for a, b in zip(y, clean))


def test_empty_views_and_missing_members():
    rope = vb.vsa2_rope_plan(64, (16, 24, 24))
    none = torch.empty(1, 2, 0, 64, dtype=BF, device="cuda")
    vb.vsa2_rope_apply(rope, none, none, grid=(1, 1, 1))
    dw = [torch.full((64,), 7.0, device="cuda") for _ in range(2)]
    ws = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    vb.vsa2_qkv_bwd(rope, (none,) * 3, (none,) * 3, (none,) * 3, None, None, *dw, ws, grid=(1, 1, 1))
    assert not dw[0].any() and not dw[1].any()
    p = Problem(1, 2, 2, (2, 3, 4), 0, 64, (16, 24, 24), vb.ROPE_PAIRS, seed=10)
    y = p.forward()
    only_k = torch.empty_like(y[1])
    vb.vsa2_qkv_fwd(p.rope, (None, p.x[1], None), (None, only_k, None), *p.w, **p.kw)
    assert torch.equal(only_k, y[1])


def test_weights_are_optional():
    p = Problem(1, 2, 2, (2, 3, 4), 0, 64, (16, 24, 24), vb.ROPE_PAIRS, seed=11)
    p.w = [torch.ones(64, device="cuda") for _ in range(2)]
    want, (dx, _) = p.forward(), p.backward()
    p.w = [None, None]
    got, (dx2, _) = p.forward(), p.backward()
    assert all(torch.equal(a, b) for a, b in zip((*want, *dx), (*got, *dx2)))


def test_another_stream_and_a_graph():
    p = Problem(1, 4, 2, (3, 8, 9), 5, 128, (44, 42, 42), vb.ROPE_PAIRS, seed=12)
    want = p.forward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = [torch.zeros_like(t) for t in want]
    side.wait_stream(torch.cuda.current_stream())
    vb.vsa2_qkv_fwd(p.rope, p.x, y, *p.w, stream=side, **p.kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(y, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.vsa2_qkv_fwd(p.rope, p.x, y, *p.w, **p.kw)
    for t in y:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(y, want))


def test_weights_at_any_fp32_address():
    p = Problem(1, 3, 3, (2, 3, 4), 0, 128, (44, 42, 42), vb.ROPE_PAIRS, seed=13)
    want, (dx, dw) = p.forward(), p.backward()
    room = torch.empty(300, device="cuda")
    for i, at in enumerate((1, 131)):
        room[at:at + 128] = p.w[i]
        p.w[i] = room[at:at + 128]
    got, (dx2, dw2) = p.forward(), p.backward()
    assert all(torch.equal(a, b) for a, b in zip((*want, *dx, *dw), (*got, *dx2, *dw2)))


@pytest.mark.parametrize("hq,hk", [(1, 3000), (3000, 1)])
def test_one_head_beside_thousands(hq, hk):
    """Each side keeps a CTA of its own."""
    p = Problem(1, hq, hk, (1, 2, 3), 0, 64, (16, 24, 24), vb.ROPE_PAIRS, seed=14)
    p.check_forward(p.forward())
    p.check_backward(*p.backward())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("dim,channels,layout", [(64, (2, 0, 4), vb.ROPE_PAIRS), (64, (16, 0, 0), vb.ROPE_HALVES), (128, (44, 42, 40), vb.ROPE_PAIRS),
                                                 (128, (32, 32, 48), vb.ROPE_HALVES), (128, (0, 0, 0), vb.ROPE_PAIRS)])
def test_what_does_not_turn_stays_as_it_is(dim, channels, layout, dtype):
    """Channels behind the last pair, and all channels of rows behind the grid: bit for bit, whatever their neighbours hold."""
    gen = torch.Generator(device="cuda").manual_seed(15)
    grid, text, total = (2, 2, 3), 5, sum(channels)
    n = 12 + text
    x = randn(gen, 2, n, 3, dim, dtype=dtype).transpose(1, 2)
    odd = torch.tensor([float("inf"), -float("inf"), -0.0, 0.0, 1.0, float("nan"), -3.0], device="cuda", dtype=dtype)
    room = x[..., total:].numel()
    x[..., total:] = odd[torch.randint(len(odd), (room,), generator=gen, device="cuda")].view(x[..., total:].shape)
    x[:, :, 12:] = odd[torch.randint(len(odd), (x[:, :, 12:].numel(),), generator=gen, device="cuda")].view(x[:, :, 12:].shape)
    rope = vb.vsa2_rope_plan(dim, channels, layout=layout)

    def same(a, b):
        bits = torch.int16 if dtype == BF else torch.int32
        return bool((a.isnan() == b.isnan()).all()) and bool(((a.contiguous().view(bits) == b.contiguous().view(bits)) | a.isnan()).all())

    for inverse in (False, True):
        y = torch.zeros_like(x)
        vb.vsa2_rope_apply(rope, x, y, grid=grid, inverse=inverse)
        assert same(y[..., total:], x[..., total:]) and same(y[:, :, 12:], x[:, :, 12:])
        assert bool(y[:, :, :12, :total].isfinite().all())
    dx = [torch.zeros_like(x) for _ in range(3)]
    vb.vsa2_qkv_bwd(rope, (x,) * 2, (x,) * 3, dx, None, None, None, None, None, norm=False, grid=grid)
    assert same(dx[0], y) and same(dx[1], y) and same(dx[2], x)


@pytest.mark.parametrize("grid", [(1, 46337, 46341), (2147483647, 1, 1), (1, 1, 2147483647), (3, 715827882, 1), (7, 17, 18046080), (65535, 181, 181), (11, 2, 3)])
def test_places_in_grids_of_any_shape(grid):
    """Rows at both ends of grids up to 2^31 - 1 tokens, as positions from the grid and as the list of the same positions."""
    gen = torch.Generator(device="cuda").manual_seed(16)
    t, h, w = grid
    rope = vb.vsa2_rope_plan(64, (16, 24, 24))
    for first in (0, max(0, min(h * w - 7, t * h * w - 37)), t * h * w - 37):
        x = randn(gen, 1, 1, 37, 64, dtype=F)
        r = torch.arange(first, first + 37, device="cuda")
        assert int(r[-1]) < t * h * w
        pos = torch.stack([r // (h * w), r // w % h, r % w], dim=-1).to(torch.int32)
        a, b = torch.empty_like(x), torch.empty_like(x)
        vb.vsa2_rope_apply(rope, x, a, grid=grid, first=first)
        vb.vsa2_rope_apply(rope, x, b, positions=pos)
        assert torch.equal(a, b)
