"""CPU-only checks of what vsa2_gate_bwd_add refuses before any CUDA call."""
import ctypes as C

import pytest

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild


@pytest.mark.parametrize("out_dtype,stride,short,dx,code", [
    (vb.BF16, 32 * 64 - 8, 0, 256, vb.ERR_INVALID_ARG),         # batch entries over one another
    (vb.BF16, -32 * 64, 0, 256, vb.ERR_INVALID_ARG),
    (vb.BF16, 32 * 64 + 4, 0, 256, vb.ERR_MISALIGNED),
    (vb.F32, 32 * 64 + 2, 0, 256, vb.ERR_MISALIGNED),
    (vb.BF16, 32 * 64, 0, 264, vb.ERR_MISALIGNED),
    (vb.BF16, 32 * 64, 0, None, vb.ERR_INVALID_ARG),
    (vb.BF16, 32 * 64, 1, 256, vb.ERR_WORKSPACE_TOO_SMALL),
])
def test_refusals(out_dtype, stride, short, dx, code):
    vbuild.build_library()
    p = vb.make_params(2, 8, 8, 64, (2, 4, 4), topk=1, out_dtype=out_dtype)
    need = vb.vsa2_gate_bwd_workspace_bytes(p, 64)
    assert vb._lib().vsa2_gate_bwd_add(C.byref(p), 64, 256, 256, 256, 256, 256, dx, stride, 256, need - short, None) == code
