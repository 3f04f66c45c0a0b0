"""GPU: more rows than a signed step of the forward's walk would hold (1,717,986,917 and more), in matrices of one column."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
ROWS = 1_750_000_001


def slices():
    """The first rows, some in the middle, those around the last row that a CTA's first, second, .. step reaches, and the last ones."""
    ctas = -(-ROWS // 4)
    return [slice(0, 1000), slice(ROWS // 2, ROWS // 2 + 1000), slice(ROWS - 1000, ROWS)] + [slice(k * ctas - 500, k * ctas + 500) for k in (1, 2, 3)]


def matrix():
    """x as a matrix of one column, with a piece of the same memory in front of it and behind it that has to stay."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    room = torch.empty(ROWS + 2048, dtype=BF, device="cuda").normal_(generator=gen)
    return room, room[1024:1024 + ROWS].view(ROWS, 1)


def test_the_norm_of_many_rows():
    _, x = matrix()
    room = torch.full((ROWS + 2048,), 7.0, dtype=BF, device="cuda")
    y = room[1024:1024 + ROWS].view(ROWS, 1)
    vb.vsa2_residual_norm_fwd(x, weight=torch.full((1,), 3.0, device="cuda"), eps=0.25, y=y)
    for s in slices():
        v = x[s].double()
        want = 3 * v / (v * v + 0.25).sqrt()
        # (one rounding to bf16, behind a handful of fp32's)
        assert ((y[s].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -18) * want.abs()).all()
    # |y| is less than 3: nothing is left of the sevens, and around the matrix nothing else
    assert int(torch.stack([(part == 7).sum() for part in y.view(-1).split(1 << 28)]).sum()) == 0
    assert (room[:1024] == 7).all() and (room[1024 + ROWS:] == 7).all()


def test_the_quantisation_of_many_rows():
    _, x = matrix()
    values = torch.full((ROWS + 64, 16), 5, dtype=torch.int8, device="cuda")
    scales = torch.full((ROWS + 64,), -1.0, device="cuda")
    vb.vsa2_int8_quantize(x, vb.Int8(values[32:32 + ROWS, :1], scales[32:32 + ROWS]))
    for s in slices():
        v, at = x[s].float().squeeze(1), slice(s.start + 32, s.stop + 32)
        assert torch.equal(values[at, 0].float(), 127 * v.sign())
        assert ((scales[at].double() - v.double().abs() / 127).abs() <= 2.0 ** -24 * v.double().abs() / 127 + 2.0 ** -106).all()
        assert (values[at, 1:] == 5).all()
    assert int(torch.stack([(part < 0).sum() for part in scales[32:32 + ROWS].split(1 << 28)]).sum()) == 0
    for edge in (slice(0, 32), slice(32 + ROWS, None)):
        assert (values[edge] == 5).all() and (scales[edge] == -1).all()
