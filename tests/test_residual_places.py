"""CPU-only: an output of the residual stream's calls that begins where another matrix of the call does is that matrix itself, or the call is refused."""
import ctypes as C

import pytest

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild

INVALID, F32, BF16 = vb.ERR_INVALID_ARG, vb.F32, vb.BF16
p = lambda s: None if s is None else C.byref(s)
N, COLS = 4, 64


@pytest.fixture(scope="module")
def lib():
    vbuild.build_library()
    return vb._lib()


def rows(address, ld=64, dtype=F32):
    return vb.Rows(address, ld, dtype, 0)


def fwd(lib, n=N, x=rows(0x1000), residual=rows(0x2000), h=None, y=None, fp8=None, int8=None):
    return lib.vsa2_residual_norm_fwd(n, COLS, p(x), p(residual), None, None, 1e-6, p(h), p(y), p(fp8), p(int8), None)


def bwd(lib, n=N, h=rows(0x1000), dy=rows(0x2000), dh=rows(0x3000), dr=None, dx=None):
    return lib.vsa2_residual_norm_bwd(n, COLS, p(h), p(dy), p(dh), None, None, 1e-6, p(dr), p(dx), None, None, 0, None)


def drop(lib, n=N, x=rows(0x1000), residual=None, y=None):
    return lib.vsa2_dropout(n, COLS, p(x), p(residual), p(vb.Drop(0x100, 0.5)), p(y), None)


# Calls that are fine go on to look for a device, which is another answer than INVALID here and on a box with one (these addresses belong to nothing, so there they are not made).
@pytest.fixture
def fine():
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up addresses")
    return lambda code: code not in (INVALID, vb.OK)


def test_an_output_in_an_input_s_place_with_another_type_or_stride(lib):
    other_ld, other_type = rows(0x1000, 72), rows(0x1000, 64, BF16)
    bf16 = rows(0x2000, 64, BF16)
    for out in (other_ld, other_type):
        assert fwd(lib, y=out) == drop(lib, y=out) == bwd(lib, dx=out) == INVALID
    assert fwd(lib, h=rows(0x1000, 72)) == fwd(lib, h=rows(0x2000, 72)) == INVALID
    assert fwd(lib, residual=bf16, h=rows(0x1000, 64, BF16)) == INVALID             # h in the place of an fp32 branch
    assert fwd(lib, y=rows(0x2000, 64, BF16)) == INVALID
    for at in (0x1000, 0x2000, 0x3000):
        assert bwd(lib, dr=rows(at, 72)) == bwd(lib, dx=rows(at, 64, BF16)) == INVALID
    assert drop(lib, residual=rows(0x2000), y=rows(0x2000, 128)) == INVALID


def test_8_bit_outputs_in_another_matrix_place(lib):
    fp8, int8 = (lambda at: vb.Fp8Matrix(at, 0x9000, 64)), (lambda at: vb.Int8Matrix(at, 0xa000, 64))
    for at in (0x1000, 0x2000, 0x3000, 0x4000):
        assert fwd(lib, h=rows(0x3000), y=rows(0x4000), fp8=fp8(at)) == INVALID
        assert fwd(lib, h=rows(0x3000), y=rows(0x4000), int8=int8(at)) == INVALID
    assert fwd(lib, fp8=fp8(0x5000), int8=int8(0x5000)) == INVALID
    assert lib.vsa2_int8_quantize(N, COLS, p(rows(0x1000)), p(int8(0x1000)), None) == INVALID


def test_an_input_itself_stays_a_valid_output(lib, fine):
    assert fine(fwd(lib, h=rows(0x2000), y=rows(0x1000))) and fine(fwd(lib, h=rows(0x1000), y=rows(0x2000)))
    assert fine(fwd(lib, x=rows(0x1000), residual=rows(0x1000), h=rows(0x1000)))
    for at in (0x1000, 0x2000, 0x3000):
        assert fine(bwd(lib, dr=rows(at))) and fine(bwd(lib, dx=rows(at)))
    assert fine(bwd(lib, dr=rows(0x3000), dx=rows(0x2000)))
    assert fine(drop(lib, y=rows(0x1000))) and fine(drop(lib, residual=rows(0x2000), y=rows(0x2000)))
    # the stride of a single row is of no use, and matrices without elements are in no place
    assert fine(fwd(lib, n=1, h=rows(0x2000, 3))) and fine(drop(lib, n=1, y=rows(0x1000, 128)))
    assert fwd(lib, n=0, y=rows(0x1000, 72)) == drop(lib, n=0, y=rows(0x1000, 64, BF16)) == vb.OK
