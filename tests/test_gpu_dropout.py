"""GPU parity of dropout: the mask bit by bit, the values with their roundings."""
import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def rng_of(seed, offset):
    wrap = lambda v: (v + 2 ** 63) % 2 ** 64 - 2 ** 63
    return torch.tensor([wrap(seed), wrap(offset)], device="cuda")


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (700, 9), (33, 1536), (5, 1531), (1, 70000), (300, 64)])
@pytest.mark.parametrize("x_type,y_type", [(BF, BF), (BF, F), (F, F), (F, BF)])
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.5, 0.999999])
def test_values(rows, cols, x_type, y_type, p):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda").to(x_type)
    r = torch.randn(rows, cols, generator=gen, device="cuda").to(y_type)
    y = torch.full((rows, cols), float("nan"), dtype=y_type, device="cuda")
    factor = ref.factors(7, 2 ** 63 + 5, rows, cols, p)
    vb.vsa2_dropout(x, y, p, rng_of(7, 2 ** 63 + 5))
    assert torch.equal(y, ref.dropped(x, factor).to(y_type))
    vb.vsa2_dropout(x, y, p, rng_of(7, 2 ** 63 + 5), residual=r)
    assert torch.equal(y, (r.float() + ref.dropped(x, factor)).to(y_type))


@pytest.mark.parametrize("seed,offset", [(0, 0), (2 ** 64 - 1, 2 ** 64 - 1), (0x299f31d0a4093822, 0x0370734413198a2e), (1, 2 ** 32), (2 ** 32, 1)])
def test_every_word_of_the_counter_and_the_key(seed, offset):
    x = torch.ones(70, 640, device="cuda")
    y = torch.empty_like(x)
    vb.vsa2_dropout(x, y, 0.5, rng_of(seed, offset))
    assert torch.equal(y.cpu().double(), ref.factors(seed, offset, 70, 640, 0.5))


def test_the_mask_does_not_depend_on_strides_types_or_the_operator():
    gen = torch.Generator(device="cuda").manual_seed(1)
    room = torch.randn(90, 1003, generator=gen, device="cuda")
    x, rng = room[:, 2:1002], rng_of(3, 9)
    y = torch.empty(90, 1000, device="cuda")
    vb.vsa2_dropout(x, y, 0.3, rng)
    whole = x.contiguous()
    vb.vsa2_dropout(whole, whole, 0.3, rng)                       # in place
    assert torch.equal(whole, y)
    h = torch.empty_like(y)
    vb.vsa2_residual_norm_fwd(x, h=h, p=0.3, rng=rng)
    assert torch.equal(h, y)
    part = torch.empty(40, 500, device="cuda")                    # a corner of it has the corner's mask
    vb.vsa2_dropout(x[:40, :500], part, 0.3, rng)
    assert torch.equal(part, y[:40, :500])
    wide = torch.full((90, 1010), 5.0, device="cuda")             # what lies behind the columns stays
    vb.vsa2_dropout(x, wide[:, 3:1003], 0.3, rng)
    assert torch.equal(wide[:, 3:1003], y) and (wide[:, :3] == 5).all() and (wide[:, 1003:] == 5).all()


def test_what_is_dropped_is_zero_whatever_it_was():
    x = torch.full((64, 512), float("inf"), device="cuda")
    x[::2] = float("nan")
    y = torch.empty_like(x)
    vb.vsa2_dropout(x, y, 0.5, rng_of(1, 1))
    kept = ref.factors(1, 1, 64, 512, 0.5).cuda() > 0
    assert (y[~kept] == 0).all() and not y[kept].isfinite().any()


def test_share_kept_and_neighbours():
    """Of n independent truth values with probability q the share is off by 6 sqrt(q (1 - q) / n) once in a billion; so are pairs of neighbours along a row and a column."""
    n = 2048 * 1536
    x = torch.ones(2048, 1536, device="cuda")
    y = torch.empty_like(x)
    vb.vsa2_dropout(x, y, 0.1, rng_of(12345, 678))
    kept = y > 0
    q = 1 - ref.threshold(0.1) / 65536
    for share, of in ((kept.double().mean(), q), ((kept[:, 1:] & kept[:, :-1]).double().mean(), q * q), ((kept[1:] & kept[:-1]).double().mean(), q * q)):
        assert abs(float(share) - of) < 6 * (of / n) ** 0.5 * 2       # (neighbouring pairs share elements: twice)


def test_a_captured_call_draws_anew():
    x = torch.ones(64, 1536, device="cuda")
    y, rng = torch.empty_like(x), rng_of(5, 0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        vb.vsa2_dropout(x, y, 0.5, rng)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            vb.vsa2_dropout(x, y, 0.5, rng)
            rng[1] += 1
    torch.cuda.synchronize()
    rng.copy_(rng_of(5, 100))
    for step in range(3):
        graph.replay()
        assert torch.equal(y.cpu().double(), ref.factors(5, 100 + step, 64, 1536, 0.5))
