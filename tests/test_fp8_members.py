"""CPU-only: an Fp8 object whose members were assigned or resized after it was made is looked at again by every call."""
import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild
from test_layer_inputs_abi import FakeTensor


def form(rows, cols):
    return (FakeTensor(torch.zeros(rows, -(-cols // 16) * 16).to(torch.float8_e4m3fn)[:, :cols]), FakeTensor(torch.zeros(-(-cols // 512), rows, 4, dtype=torch.uint8)))


CHANGES = [
    lambda f: setattr(f, "scales", FakeTensor(torch.zeros(1, 5, 4, dtype=torch.uint8))),                # too short
    lambda f: setattr(f, "scales", FakeTensor(torch.zeros(1, 6, 4))),                                   # another type
    lambda f: setattr(f, "scales", FakeTensor(torch.zeros(24, dtype=torch.uint8))),
    lambda f: setattr(f, "scales", FakeTensor(torch.zeros(4, 6, 1, dtype=torch.uint8).transpose(0, 2))),  # right shape, other order
    lambda f: setattr(f, "values", form(6, 513)[0]),                                                    # more blocks than scales
    lambda f: setattr(f, "values", form(7, 40)[0]),
    lambda f: setattr(f, "values", FakeTensor(torch.zeros(6, 48, dtype=torch.uint8)[:, :40])),
    lambda f: setattr(f, "values", FakeTensor(torch.zeros(40, 16).to(torch.float8_e4m3fn)[:, :6].T)),     # columns contiguous
    lambda f: setattr(f, "values", torch.zeros(6, 48).to(torch.float8_e4m3fn)[:, :40]),                  # host memory
    lambda f: setattr(f.scales, "shape", torch.Size((1, 5, 4))),                                        # resized in place
]


@pytest.mark.parametrize("change", CHANGES)
def test_changed_members_are_refused(change, monkeypatch):
    vbuild.build_library()
    called = []
    types = (torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn, torch.uint8)
    import ctypes as C
    noted = C.CFUNCTYPE(C.c_int)(lambda: called.append(1) or 0)      # (in the place of all five functions: nothing of the library runs)
    address = C.cast(noted, C.c_void_p).value
    m, lib = vb._marshal(), vb._lib()
    real = tuple(C.cast(f, C.c_void_p).value for f in (lib.vsa2_rope_apply, lib.vsa2_qkv_fwd, lib.vsa2_qkv_bwd, lib.vsa2_fp8_quantize, lib.vsa2_fp8_matmul))
    m.bind(types, (address,) * 5, lambda s: 7)
    try:
        x, c, ws = FakeTensor(torch.zeros(6, 40)), FakeTensor(torch.zeros(6, 7)), FakeTensor(torch.zeros(100))
        good = vb.Fp8(*form(6, 40))
        vb.vsa2_fp8_quantize(x, good)
        vb.vsa2_fp8_matmul(good, vb.Fp8(*form(7, 40)), c, ws)
        assert len(called) == 2
        changed = vb.Fp8(*form(6, 40))
        change(changed)
        with pytest.raises(ValueError):
            vb.vsa2_fp8_quantize(x, changed)
        with pytest.raises(ValueError):
            vb.vsa2_fp8_matmul(changed, vb.Fp8(*form(7, 40)), c, ws)
        assert len(called) == 2
    finally:
        m.bind(types, real, vb._stream)


@pytest.mark.parametrize("rows,cols", [(0, 8), (8, 0), (0, 0), (1, 1), (3, 600)])
def test_dequantized_shapes(rows, cols):
    f = vb.Fp8.empty(rows, cols, device="cpu")
    f.values.copy_(torch.full((rows, cols), 1.5).to(torch.float8_e4m3fn))
    f.scales.fill_(128)
    x = f.dequantize()
    assert x.shape == (rows, cols) and (x == 3.0).all()
