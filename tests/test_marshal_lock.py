"""CPU-only: the calls that the C module marshals run without the interpreter's lock, as those through ctypes do."""
import ctypes as C
import shutil
import subprocess
import threading

import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild
from test_layer_inputs_abi import FakeTensor

# waits (two seconds at most) for what only another thread of Python does
SOURCE = """
#include <unistd.h>
volatile int entered, answered;
int waits(void) {
  entered = 1;
  for (int i = 0; i < 2000; ++i) {
    if (answered) return -41;
    usleep(1000);
  }
  return -42;
}
"""


@pytest.fixture(scope="module")
def waiting(tmp_path_factory):
    vbuild.build_library()
    at = tmp_path_factory.mktemp("waits")
    (at / "waits.c").write_text(SOURCE)
    subprocess.check_call([shutil.which("gcc") or "cc", "-shared", "-fPIC", "-o", str(at / "waits.so"), str(at / "waits.c")])
    lib = C.CDLL(str(at / "waits.so"))
    types, real = (torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn, torch.uint8), vb._lib()
    fns = tuple(C.cast(f, C.c_void_p).value for f in (real.vsa2_rope_apply, real.vsa2_qkv_fwd, real.vsa2_qkv_bwd, real.vsa2_fp8_quantize, real.vsa2_fp8_matmul))
    m = vb._marshal()
    m.bind(types, (C.cast(lib.waits, C.c_void_p).value,) * 5, lambda s: 7)
    yield lib
    m.bind(types, fns, vb._stream)


def f8(rows, cols):
    return vb.Fp8(FakeTensor(torch.zeros(rows, -(-cols // 16) * 16).to(torch.float8_e4m3fn)[:, :cols]), FakeTensor(torch.zeros(-(-cols // 512), rows, 4, dtype=torch.uint8)))


@pytest.mark.parametrize("name", ["rope_apply", "qkv_fwd", "qkv_bwd", "fp8_quantize", "fp8_matmul"])
def test_another_thread_runs_while_a_call_waits(waiting, name):
    entered, answered = (C.c_int.in_dll(waiting, n) for n in ("entered", "answered"))
    entered.value = answered.value = 0
    rope, x = vb.vsa2_rope_plan(64, (16, 24, 24)), FakeTensor(torch.zeros(1, 2, 5, 64))
    w = [FakeTensor(torch.zeros(64)) for _ in range(4)]
    ws = FakeTensor(torch.zeros(100))
    call = {"rope_apply": lambda: vb.vsa2_rope_apply(rope, x, x, grid=(1, 1, 5)),
            "qkv_fwd": lambda: vb.vsa2_qkv_fwd(rope, (x,) * 3, (x,) * 3, *w[:2], grid=(1, 1, 5)),
            "qkv_bwd": lambda: vb.vsa2_qkv_bwd(rope, (x,) * 3, (x,) * 3, (x,) * 3, *w, ws, grid=(1, 1, 5)),
            "fp8_quantize": lambda: vb.vsa2_fp8_quantize(FakeTensor(torch.zeros(6, 40)), f8(6, 40)),
            "fp8_matmul": lambda: vb.vsa2_fp8_matmul(f8(6, 40), f8(7, 40), FakeTensor(torch.zeros(6, 7)), ws)}[name]

    def answer():
        while not entered.value:
            pass
        answered.value = 1

    thread = threading.Thread(target=answer)
    thread.start()
    try:
        with pytest.raises(vb.Vsa2Error) as e:
            call()
        assert e.value.code == -41          # (-42: nobody could answer)
    finally:
        entered.value = 1
        thread.join()
