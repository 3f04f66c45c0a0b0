"""CPU-only checks of the residual stream's calls: what the C functions and the binding refuse, and the generator of the tests against published answers."""
import ctypes as C

import numpy as np
import pytest
import torch

import residual_reference as ref
from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild

INVALID, UNSUPPORTED, SMALL, MISALIGNED = vb.ERR_INVALID_ARG, vb.ERR_UNSUPPORTED, vb.ERR_WORKSPACE_TOO_SMALL, vb.ERR_MISALIGNED


@pytest.fixture(scope="module")
def lib():
    vbuild.build_library()
    return vb._lib()


def test_the_generator_gives_the_published_answers():
    """The known answers that come with the generator's publication, for Philox 4x32 with ten rounds."""
    for counter, key, want in (((0,) * 4, (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(v) for v in ref.philox(counter, key)) == want


def test_the_mask_takes_sixteen_bits_of_each_word():
    words = ref.philox([np.array([3]), np.array([2]), np.array([11]), np.array([0])], (5, 0))
    bits = [int(w[0]) >> s & 0xffff for w in words for s in (0, 16)]
    t = ref.threshold(0.5)
    assert ref.factors(5, 11, 3, 32, 0.5)[2, 24:].tolist() == [2.0 if b >= t else 0.0 for b in bits]


at = lambda address: C.c_void_p(address)
F32, BF16 = vb.F32, vb.BF16


def rows(address=0x1000, ld=64, dtype=F32):
    return vb.Rows(address, ld, dtype, 0)


def fwd(lib, n=4, cols=64, x=rows(), residual=None, drop=None, weight=None, eps=1e-6, h=rows(0x2000), y=None, fp8=None, int8=None):
    p = lambda s: None if s is None else C.byref(s)
    return lib.vsa2_residual_norm_fwd(n, cols, p(x), p(residual), p(drop), weight, eps, p(h), p(y), p(fp8), p(int8), None)


def test_forward_refusals(lib):
    assert fwd(lib, n=-1) == fwd(lib, cols=-1) == fwd(lib, x=None) == fwd(lib, h=None) == INVALID      # (the last: nothing is wanted)
    assert fwd(lib, eps=-1.0) == fwd(lib, eps=float("nan")) == INVALID
    assert fwd(lib, x=rows(0)) == fwd(lib, x=rows(ld=63)) == fwd(lib, x=rows(dtype=2)) == INVALID
    assert fwd(lib, residual=rows(dtype=BF16)) == INVALID                       # h has the residual's type
    assert fwd(lib, x=rows(dtype=BF16)) == INVALID                              # or x's
    assert fwd(lib, y=rows(0x2000)) == INVALID                                  # two outputs in one place
    assert fwd(lib, x=rows(0x1002)) == fwd(lib, h=rows(0x2001)) == fwd(lib, weight=at(0x3001)) == MISALIGNED
    assert fwd(lib, fp8=vb.Fp8Matrix(0x4000, 0x5000, 32)) == INVALID and fwd(lib, fp8=vb.Fp8Matrix(0x4008, 0x5000, 64)) == MISALIGNED
    assert fwd(lib, int8=vb.Int8Matrix(0x4000, 0x5000, 48)) == fwd(lib, int8=vb.Int8Matrix(None, 0x5000, 64)) == fwd(lib, int8=vb.Int8Matrix(0x4000, None, 64)) == INVALID
    assert fwd(lib, int8=vb.Int8Matrix(0x4008, 0x5000, 64)) == fwd(lib, int8=vb.Int8Matrix(0x4000, 0x5000, 72)) == fwd(lib, int8=vb.Int8Matrix(0x4000, 0x5002, 64)) == MISALIGNED
    assert fwd(lib, cols=(1 << 22) + 1, x=rows(ld=1 << 23), h=rows(0x2000, 1 << 23)) == UNSUPPORTED
    for p in (-0.1, 1.0, 2.0, float("nan"), float("inf")):
        assert fwd(lib, drop=vb.Drop(0x100, p)) == INVALID
    assert fwd(lib, drop=vb.Drop(None, 0.1)) == INVALID and fwd(lib, drop=vb.Drop(0x104, 0.1)) == MISALIGNED
    assert fwd(lib, n=0) == fwd(lib, cols=0) == vb.OK


def bwd(lib, n=4, cols=64, h=rows(), dy=rows(0x2000), dh=None, drop=None, weight=None, eps=1e-6, dr=rows(0x3000), dx=None, dw=None, ws=None, size=0):
    p = lambda s: None if s is None else C.byref(s)
    return lib.vsa2_residual_norm_bwd(n, cols, p(h), p(dy), p(dh), p(drop), weight, eps, p(dr), p(dx), dw, ws, size, None)


def test_backward_refusals(lib):
    need = vb.vsa2_residual_norm_bwd_workspace_bytes(4, 64)
    assert need >= 4 * 64 * 4 and need % 256 == 0
    assert bwd(lib, h=None) == bwd(lib, dy=None) == bwd(lib, dr=None) == bwd(lib, n=-1) == bwd(lib, eps=-1.0) == INVALID
    assert bwd(lib, dh=rows(0x4000, dtype=BF16)) == bwd(lib, dr=rows(0x3000, dtype=BF16)) == bwd(lib, dx=rows(0x3000)) == INVALID
    assert bwd(lib, dw=at(0x5000)) == INVALID
    assert bwd(lib, dw=at(0x5000), ws=at(0x6010), size=need) == bwd(lib, dw=at(0x5002), ws=at(0x6000), size=need) == MISALIGNED
    assert bwd(lib, dw=at(0x5000), ws=at(0x6000), size=need - 1) == SMALL
    assert bwd(lib, drop=vb.Drop(0x100, 1.0)) == INVALID
    assert bwd(lib, cols=0) == bwd(lib, n=0) == vb.OK


def test_workspaces_grow_with_every_size():
    for a, b in (((1, 1), (2, 1)), ((100, 64), (100, 65)), ((1184, 1536), (5000, 1536)), ((5000, 1536), (75600, 5120))):
        assert vb.vsa2_residual_norm_bwd_workspace_bytes(*a) <= vb.vsa2_residual_norm_bwd_workspace_bytes(*b)
    assert vb.vsa2_residual_norm_bwd_workspace_bytes(-1, 4) == 0 and vb.vsa2_int8_matmul_workspace_bytes(1, -1, 4) == 0
    import itertools
    import random
    rng = random.Random(3)
    sizes = [tuple(int(2 ** rng.uniform(0, e)) for e in (16, 14, 15)) for _ in range(60)]
    for a, b in itertools.combinations(sizes, 2):
        if all(x <= y for x, y in zip(a, b)):
            assert vb.vsa2_int8_matmul_workspace_bytes(*a) <= vb.vsa2_int8_matmul_workspace_bytes(*b)


def test_dropout_and_quantisation_refusals(lib):
    p = lambda s: None if s is None else C.byref(s)
    drop = lambda x=rows(), r=None, d=vb.Drop(0x100, 0.5), y=rows(0x2000), n=4, cols=64: lib.vsa2_dropout(n, cols, p(x), p(r), p(d), p(y), None)
    assert drop(x=None) == drop(y=None) == drop(d=None) == drop(r=rows(0x3000, dtype=BF16)) == drop(d=vb.Drop(0x100, 1.0)) == drop(y=rows(0x2000, ld=8)) == INVALID
    assert drop(y=rows(0x2002)) == drop(d=vb.Drop(0x101, 0.5)) == MISALIGNED
    assert drop(n=0) == drop(cols=0) == vb.OK
    quantize = lambda x=rows(), out=vb.Int8Matrix(0x2000, 0x3000, 64), n=4, cols=64: lib.vsa2_int8_quantize(n, cols, p(x), p(out), None)
    assert quantize(x=None) == quantize(out=None) == quantize(n=-1) == quantize(x=rows(ld=1)) == quantize(out=vb.Int8Matrix(0x2000, 0x3000, 32)) == INVALID
    assert quantize(out=vb.Int8Matrix(0x2001, 0x3000, 64)) == quantize(x=rows(0x1001)) == MISALIGNED
    assert quantize(n=0) == vb.OK


def test_product_refusals(lib):
    p = lambda s: None if s is None else C.byref(s)
    need = vb.vsa2_int8_matmul_workspace_bytes(4, 64, 128)
    ok = dict(m=4, n=64, k=128, a=vb.Int8Matrix(0x1000, 0x2000, 128), b=vb.Int8Matrix(0x3000, 0x4000, 128), bias=None, c=at(0x5000), dtype=F32, ldc=64, ws=at(0x6000), size=need)

    def call(**kw):
        v = {**ok, **kw}
        return lib.vsa2_int8_matmul(v["m"], v["n"], v["k"], p(v["a"]), p(v["b"]), v["bias"], v["c"], v["dtype"], v["ldc"], v["ws"], v["size"], None)

    assert call(m=-1) == call(a=None) == call(b=None) == call(c=None) == call(ws=None) == call(dtype=5) == call(ldc=63) == INVALID
    assert call(a=vb.Int8Matrix(0x1000, None, 128)) == call(b=vb.Int8Matrix(0x3000, 0x4000, 112)) == INVALID
    assert call(c=at(0x5002)) == call(bias=at(0x7001)) == call(ws=at(0x6080)) == call(a=vb.Int8Matrix(0x1008, 0x2000, 128)) == call(b=vb.Int8Matrix(0x3000, 0x4000, 136)) == MISALIGNED
    assert call(size=need - 1) == SMALL
    assert call(k=131072, a=vb.Int8Matrix(0x1000, 0x2000, 131072), b=vb.Int8Matrix(0x3000, 0x4000, 131072), size=1 << 40) == UNSUPPORTED
    assert call(m=0) == call(n=0) == vb.OK


def test_the_binding_refuses_what_it_cannot_marshal():
    vbuild.build_library()
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="CUDA"):
        vb.vsa2_residual_norm_fwd(x, h=x)
    with pytest.raises(ValueError, match="CUDA"):
        vb.vsa2_dropout(x, x, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="int8"):
        vb.Int8(x, x[:, 0])
    with pytest.raises(ValueError, match="rows"):
        vb.Int8(x.to(torch.int8), torch.zeros(5))
    with pytest.raises(ValueError, match="CUDA"):
        vb.vsa2_int8_quantize(x, vb.Int8.empty(4, 64, "cpu"))
    with pytest.raises(ValueError, match="CUDA"):
        vb.vsa2_int8_matmul(vb.Int8.empty(4, 64, "cpu"), vb.Int8.empty(8, 64, "cpu"), torch.zeros(4, 8), torch.zeros(256, dtype=torch.uint8))
    assert vb.Int8.empty(3, 50, "cpu").values.stride() == (64, 1)
