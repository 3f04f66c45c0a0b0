"""CPU-only checks of the entry points between hidden states and attention: the rotation's plan, and what each call refuses before any CUDA call."""
import ctypes as C
import math

import pytest
import torch

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild


@pytest.fixture(scope="module", autouse=True)
def lib():
    vbuild.build_library()
    return vb._lib()


def heads(data=256, batch=2, heads=3, tokens=5, channels=64, dtype=vb.BF16, strides=None):
    sb, sh, st = strides or (heads * tokens * channels, tokens * channels, channels)
    return vb.Heads(data, sb, sh, st, batch, heads, tokens, channels, dtype, 0)


def place(**kw):
    p = vb.Place(1, 1, 5, 0, None, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_plan_holds_the_frequencies_as_fractions_of_a_turn():
    channels, theta, scale = (44, 42, 42), (1e4, 500.0, 1e6), (1.0, 0.5, -2.0)
    for layout in (vb.ROPE_PAIRS, vb.ROPE_HALVES):
        plan = vb.vsa2_rope_plan(128, channels, theta=theta, scale=scale, layout=layout)
        assert list(plan.axis_pairs) == [22, 21, 21] and plan.head_dim == 128 and plan.layout == layout
        p = 0
        for a, c in enumerate(channels):
            for j in range(c // 2):
                want = scale[a] * theta[a] ** (-2.0 * j / c) / (2 * math.pi) % 1.0
                assert abs(plan.turn[p] / 2.0 ** 64 - want) <= 2.0 ** -50        # (the check's own 64-bit rounding)
                p += 1
        assert p == 64


def test_plan_is_exact_where_the_fraction_is_known():
    """Positions that turn by whole turns: scale 2 pi is not a 64-bit number, but its nearest one is 2^-52 off at most."""
    plan = vb.vsa2_rope_plan(64, (0, 0, 2), scale=math.pi / 2)
    assert abs(plan.turn[0] - (1 << 62)) <= 1 << 10
    assert vb.vsa2_rope_plan(64, (0, 0, 64), scale=0.0).turn[5] == 0
    assert list(vb.vsa2_rope_plan(64, (0, 0, 0)).axis_pairs) == [0, 0, 0]


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=96, channels=(32, 32, 32)), vb.ERR_UNSUPPORTED),
    (dict(head_dim=64, channels=(16, 24, 23)), vb.ERR_INVALID_ARG),                    # odd
    (dict(head_dim=64, channels=(16, 26, 24)), vb.ERR_INVALID_ARG),                    # more than the head has
    (dict(head_dim=64, channels=(-2, 24, 24)), vb.ERR_INVALID_ARG),
    (dict(head_dim=64, channels=(2, 24, 24), layout=vb.ROPE_HALVES), vb.ERR_UNSUPPORTED),
    (dict(head_dim=64, channels=(16, 24, 24), layout=2), vb.ERR_INVALID_ARG),
    (dict(head_dim=64, channels=(16, 24, 24), theta=0.0), vb.ERR_INVALID_ARG),
    (dict(head_dim=64, channels=(16, 24, 24), theta=float("inf")), vb.ERR_INVALID_ARG),
    (dict(head_dim=64, channels=(16, 24, 24), scale=(1.0, float("nan"), 1.0)), vb.ERR_INVALID_ARG),
])
def test_plan_refusals(kw, code):
    with pytest.raises(vb.Vsa2Error) as e:
        vb.vsa2_rope_plan(**kw)
    assert e.value.code == code
    with pytest.raises(ValueError):
        vb.vsa2_rope_plan(64, (32, 32))


@pytest.mark.parametrize("x,y,where,code", [
    (dict(data=None), {}, {}, vb.ERR_INVALID_ARG),
    (dict(data=264), {}, {}, vb.ERR_MISALIGNED),
    (dict(strides=(960, 320, 68)), {}, {}, vb.ERR_MISALIGNED),                         # rows not on 16 bytes
    ({}, dict(strides=(960, 320, 68)), {}, vb.ERR_MISALIGNED),
    (dict(channels=32), dict(channels=32), {}, vb.ERR_UNSUPPORTED),
    (dict(channels=128), dict(channels=128), {}, vb.ERR_INVALID_ARG),                  # not the plan's
    (dict(heads=2), {}, {}, vb.ERR_INVALID_ARG),                                       # shapes differ
    (dict(tokens=-1), dict(tokens=-1), {}, vb.ERR_INVALID_ARG),
    (dict(dtype=2), {}, {}, vb.ERR_INVALID_ARG),
    ({}, dict(strides=(960, 0, 64)), {}, vb.ERR_INVALID_ARG),                          # heads written over one another
    ({}, {}, dict(grid_w=0), vb.ERR_INVALID_ARG),
    ({}, {}, dict(first=-1), vb.ERR_INVALID_ARG),
    ({}, {}, dict(grid_h=1 << 20, grid_w=1 << 20), vb.ERR_UNSUPPORTED),
    ({}, {}, dict(positions=258), vb.ERR_MISALIGNED),
    ({}, {}, dict(positions=256, positions_batch_stride=-15), vb.ERR_INVALID_ARG),
])
def test_rotation_refusals(lib, x, y, where, code):
    rope = vb.vsa2_rope_plan(64, (16, 24, 24))
    assert lib.vsa2_rope_apply(C.byref(rope), C.byref(place(**where)), C.byref(heads(**x)), C.byref(heads(**y)), 0, None) == code


def test_null_structs_are_refused(lib):
    rope, at, v = vb.vsa2_rope_plan(64, (16, 24, 24)), place(), heads()
    full = [C.byref(rope), C.byref(at), C.byref(v), C.byref(v), 0, None]
    for i in range(4):
        args = list(full)
        args[i] = None
        assert lib.vsa2_rope_apply(*args) == vb.ERR_INVALID_ARG
    three = (vb.Heads * 3)(v, v, v)
    assert lib.vsa2_qkv_fwd(C.byref(rope), C.byref(at), None, None, three, None) == vb.ERR_INVALID_ARG
    assert lib.vsa2_qkv_fwd(C.byref(rope), None, None, three, three, None) == vb.ERR_INVALID_ARG
    assert lib.vsa2_fp8_quantize(256, vb.BF16, 1, 1, 1, 0, None, None, None) == vb.ERR_INVALID_ARG
    assert lib.vsa2_rope_plan(64, 0, None, None, None, None) == vb.ERR_INVALID_ARG


def test_damaged_plans_are_refused(lib):
    v = heads()
    for change in (dict(layout=3), dict(head_dim=128), dict(axis_pairs=(20, 20, 20)), dict(axis_pairs=(-1, 2, 2))):
        rope = vb.vsa2_rope_plan(64, (16, 24, 24))
        for k, val in change.items():
            setattr(rope, k, (C.c_int32 * 3)(*val) if k == "axis_pairs" else val)
        assert lib.vsa2_rope_apply(C.byref(rope), C.byref(place()), C.byref(v), C.byref(v), 0, None) == vb.ERR_INVALID_ARG


def test_norm_and_gradient_refusals(lib):
    rope, at = vb.vsa2_rope_plan(64, (16, 24, 24)), place()
    three, two = (vb.Heads * 3)(heads(), heads(), heads()), (vb.Heads * 2)(heads(), heads())
    norm = vb.QkNorm(256, 256, 1e-6, 0)
    need = vb.vsa2_qkv_bwd_workspace_bytes(64)
    assert need > 0 and vb.vsa2_qkv_bwd_workspace_bytes(96) == 0

    def bwd(norm=norm, x=two, dy=three, dx=three, ws=256, nbytes=need):
        return lib.vsa2_qkv_bwd(C.byref(rope), C.byref(at), C.byref(norm), x, dy, dx, 256, 256, ws, nbytes, None)

    assert bwd(nbytes=need - 1) == vb.ERR_WORKSPACE_TOO_SMALL
    assert bwd(ws=128) == vb.ERR_MISALIGNED
    assert bwd(ws=None) == vb.ERR_INVALID_ARG
    assert bwd(x=None) == vb.ERR_INVALID_ARG
    assert bwd(norm=vb.QkNorm(256, 256, -1.0, 0)) == vb.ERR_INVALID_ARG
    assert bwd(norm=vb.QkNorm(256, 256, float("nan"), 0)) == vb.ERR_INVALID_ARG
    assert bwd(x=(vb.Heads * 2)(heads(), heads(heads=2))) == vb.ERR_INVALID_ARG
    assert bwd(dy=(vb.Heads * 3)(heads(), heads(), heads(dtype=vb.F32))) == vb.ERR_INVALID_ARG       # one type for a side
    assert bwd(dx=(vb.Heads * 3)(heads(), heads(tokens=4), heads())) == vb.ERR_INVALID_ARG
    assert lib.vsa2_qkv_fwd(C.byref(rope), C.byref(at), C.byref(vb.QkNorm(256, 256, -1.0, 0)), three, three, None) == vb.ERR_INVALID_ARG


@pytest.mark.parametrize("q_weight,k_weight,d_q_weight,d_k_weight", [(258, 256, 256, 256), (256, 257, 256, 256), (256, 256, 258, 256), (256, 256, 256, 259)])
def test_weights_off_their_type_are_refused(lib, q_weight, k_weight, d_q_weight, d_k_weight):
    rope, at, norm = vb.vsa2_rope_plan(64, (16, 24, 24)), place(), vb.QkNorm(q_weight, k_weight, 1e-6, 0)
    three, two = (vb.Heads * 3)(heads(), heads(), heads()), (vb.Heads * 2)(heads(), heads())
    need = vb.vsa2_qkv_bwd_workspace_bytes(64)
    assert lib.vsa2_qkv_bwd(C.byref(rope), C.byref(at), C.byref(norm), two, three, three, d_q_weight, d_k_weight, 256, need, None) == vb.ERR_MISALIGNED
    if q_weight % 4 or k_weight % 4:
        assert lib.vsa2_qkv_fwd(C.byref(rope), C.byref(at), C.byref(norm), three, three, None) == vb.ERR_MISALIGNED


def test_more_heads_than_a_call_takes_are_refused(lib):
    """Three views whose heads together pass 32 bits, and one head more than a call takes."""
    rope, at = vb.vsa2_rope_plan(64, (16, 24, 24)), place()
    for n in ((1 << 30,) * 3, (1 << 20, 1, 0)):
        three = (vb.Heads * 3)(*(heads(batch=1, heads=h, tokens=1) for h in n))
        assert lib.vsa2_qkv_fwd(C.byref(rope), C.byref(at), None, three, three, None) == vb.ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), vb.ERR_INVALID_ARG),
    (dict(x=None), vb.ERR_INVALID_ARG),
    (dict(x=257), vb.ERR_MISALIGNED),
    (dict(ld=99), vb.ERR_INVALID_ARG),
    (dict(dtype=5), vb.ERR_INVALID_ARG),
    (dict(cols=1 << 23, ld=1 << 23), vb.ERR_UNSUPPORTED),
    (dict(out=(0, 256, 112)), vb.ERR_INVALID_ARG),
    (dict(out=(256, 256, 96)), vb.ERR_INVALID_ARG),          # rows shorter than the columns
    (dict(out=(256, 256, 104)), vb.ERR_MISALIGNED),          # rows not on 16 bytes
    (dict(out=(264, 256, 112)), vb.ERR_MISALIGNED),
    (dict(out=(256, 258, 112)), vb.ERR_MISALIGNED),
])
def test_quantize_refusals(lib, kw, code):
    a = dict(x=256, dtype=vb.BF16, rows=10, cols=100, ld=100, out=(256, 256, 112))
    a.update(kw)
    out = vb.Fp8Matrix(*a["out"])
    assert lib.vsa2_fp8_quantize(a["x"], a["dtype"], a["rows"], a["cols"], a["ld"], 0, C.byref(out), None, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), vb.ERR_INVALID_ARG),
    (dict(c=None), vb.ERR_INVALID_ARG),
    (dict(c=257), vb.ERR_MISALIGNED),
    (dict(ldc=299), vb.ERR_INVALID_ARG),
    (dict(c_dtype=7), vb.ERR_INVALID_ARG),
    (dict(a=(256, 256, 128)), vb.ERR_INVALID_ARG),
    (dict(b=(256, 256, 200)), vb.ERR_MISALIGNED),
    (dict(b=(8, 256, 208)), vb.ERR_MISALIGNED),
    (dict(a=(256, 0, 208)), vb.ERR_INVALID_ARG),
    (dict(ws=None), vb.ERR_INVALID_ARG),
    (dict(ws=128), vb.ERR_MISALIGNED),
    (dict(short=1), vb.ERR_WORKSPACE_TOO_SMALL),
    (dict(m=1 << 30, n=1 << 20, ldc=1 << 20), vb.ERR_UNSUPPORTED),
])
def test_product_refusals(lib, kw, code):
    a = dict(m=20, n=300, k=200, a=(256, 256, 208), b=(256, 256, 208), c=256, c_dtype=vb.BF16, ldc=300, ws=256, short=0)
    a.update(kw)
    need = vb.vsa2_fp8_matmul_workspace_bytes(20, 300, 200)
    assert lib.vsa2_fp8_matmul(a["m"], a["n"], a["k"], C.byref(vb.Fp8Matrix(*a["a"])), C.byref(vb.Fp8Matrix(*a["b"])), a["c"], a["c_dtype"],
                               a["ldc"], a["ws"], need - a["short"], None) == code


def test_sizes_of_zero_need_no_device(lib):
    rope, at = vb.vsa2_rope_plan(64, (16, 24, 24)), place()
    for kw in (dict(tokens=0), dict(batch=0), dict(heads=0)):
        v = heads(data=None, **kw)
        assert lib.vsa2_rope_apply(C.byref(rope), C.byref(at), C.byref(v), C.byref(v), 0, None) == vb.OK
    f = vb.Fp8Matrix(256, 256, 208)
    assert lib.vsa2_fp8_matmul(0, 300, 200, C.byref(f), C.byref(f), 256, vb.BF16, 300, 256, 1 << 30, None) == vb.OK
    assert lib.vsa2_fp8_quantize(None, vb.BF16, 0, 100, 100, 0, C.byref(f), None, None) == vb.OK


def test_binding_refuses_what_it_cannot_marshal():
    rope = vb.vsa2_rope_plan(64, (16, 24, 24))
    with pytest.raises(ValueError):
        vb.vsa2_rope_apply(rope, torch.zeros(1, 1, 4, 64), torch.zeros(1, 1, 4, 64), grid=(1, 1, 4))      # host tensors
    with pytest.raises(ValueError):
        vb.Fp8(torch.zeros(4, 4), torch.zeros(1, 4, 4, dtype=torch.uint8))
    with pytest.raises(ValueError):
        vb.Fp8(torch.zeros(4, 4).to(torch.float8_e4m3fn), torch.zeros(1, 4, 1, dtype=torch.uint8))
    f = vb.Fp8.empty(4, 20, device="cpu")
    assert f.shape == (4, 20) and f.values.stride(0) == 32
    with pytest.raises(ValueError):
        vb.vsa2_fp8_quantize(torch.zeros(4, 20), f)
    with pytest.raises(ValueError):
        vb.vsa2_fp8_matmul(f, vb.Fp8.empty(4, 21, device="cpu"), torch.zeros(4, 4), None)
    with pytest.raises(ValueError):
        vb.Fp8(torch.zeros(4, 20).to(torch.float8_e4m3fn), torch.zeros(1, 4, 4))
    with pytest.raises(ValueError):
        vb.Fp8(torch.zeros(4).to(torch.float8_e4m3fn), torch.zeros(1, 4, 4, dtype=torch.uint8))
    with pytest.raises(AttributeError):
        vb.vsa2_rope_apply(rope, "x", "y", grid=(1, 1, 4))
    with pytest.raises(TypeError):
        vb._marshal().rope_apply(rope)
    with pytest.raises(ValueError):
        vb.vsa2_qkv_fwd(rope, (None, None, None), (None, None, None), grid=(1, 1, 4))
    with pytest.raises(ValueError):
        vb.vsa2_qkv_fwd(rope, (None,), (None,), grid=(1, 1, 4))


class FakeTensor:
    """What the marshalling asks of a CUDA tensor; nothing is ever launched with it."""

    def __init__(self, tensor, is_cuda=True):
        self._t, self.shape, self.dtype, self.is_cuda, self.nbytes = tensor, tensor.shape, tensor.dtype, is_cuda, tensor.nbytes

    def __getattr__(self, name):
        return getattr(self._t, name)


def test_marshalling_passes_what_the_tensors_say(monkeypatch):
    """Bound to functions that record their arguments instead of the library's."""
    seen = {}
    rope_t = C.CFUNCTYPE(C.c_int, C.POINTER(vb.Rope), C.POINTER(vb.Place), C.POINTER(vb.Heads), C.POINTER(vb.Heads), C.c_int32, C.c_void_p)
    fwd_t = C.CFUNCTYPE(C.c_int, C.POINTER(vb.Rope), C.POINTER(vb.Place), C.POINTER(vb.QkNorm), C.POINTER(vb.Heads), C.POINTER(vb.Heads), C.c_void_p)
    bwd_t = C.CFUNCTYPE(C.c_int, C.POINTER(vb.Rope), C.POINTER(vb.Place), C.POINTER(vb.QkNorm), *[C.POINTER(vb.Heads)] * 3, *[C.c_void_p] * 3, C.c_size_t,
                        C.c_void_p)
    qz_t = C.CFUNCTYPE(C.c_int, C.c_void_p, *[C.c_int32] * 3, C.c_int64, C.c_int32, C.POINTER(vb.Fp8Matrix), C.POINTER(vb.Fp8Matrix), C.c_void_p)
    mm_t = C.CFUNCTYPE(C.c_int, *[C.c_int32] * 3, C.POINTER(vb.Fp8Matrix), C.POINTER(vb.Fp8Matrix), C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_size_t,
                       C.c_void_p)
    fields = lambda s: {f: (list(getattr(s, f)) if f in ("turn", "axis_pairs") else getattr(s, f)) for f, _ in s._fields_}
    view = lambda s: tuple(fields(s).values())

    def keep(name, *indices):
        def f(*a):
            seen[name] = [x if not isinstance(x, C._Pointer) else [view(x[k]) for k in range(indices[i])] if x else None for i, x in enumerate(a)]
            return 0
        return f

    fns = (rope_t(keep("rope", 1, 1, 1, 1, 0, 0)), fwd_t(keep("fwd", 1, 1, 1, 3, 3, 0)), bwd_t(keep("bwd", 1, 1, 1, 2, 3, 3, 0, 0, 0, 0, 0)),
           qz_t(keep("qz", 0, 0, 0, 0, 0, 0, 1, 1, 0)), mm_t(keep("mm", 0, 0, 0, 1, 1, 0, 0, 0, 0, 0, 0)))
    types = (torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn, torch.uint8)
    m = vb._marshal()
    lib = vb._lib()
    real = tuple(C.cast(f, C.c_void_p).value for f in (lib.vsa2_rope_apply, lib.vsa2_qkv_fwd, lib.vsa2_qkv_bwd, lib.vsa2_fp8_quantize, lib.vsa2_fp8_matmul))
    m.bind(types, tuple(C.cast(f, C.c_void_p).value for f in fns), lambda s: 77 if s is None else s)
    try:
        rope = vb.vsa2_rope_plan(64, (16, 24, 24))
        base = torch.zeros(2, 5, 7, 64, dtype=torch.bfloat16)
        x, y = FakeTensor(base.transpose(1, 2)[:, 2:5]), FakeTensor(torch.zeros(2, 3, 5, 64))
        pos = FakeTensor(torch.zeros(2, 5, 3, dtype=torch.int32))
        vb.vsa2_rope_apply(rope, x, y, grid=(1, 2, 3), first=4, inverse=True, stream=9)
        r, p, vx, vy, inverse, stream = seen["rope"]
        assert r[0][-1] == list(rope.turn) and p == [(1, 2, 3, 4, None, 0)] and (inverse, stream) == (1, 9)
        assert vx == [(x.data_ptr(), 5 * 7 * 64, 64, 7 * 64, 2, 3, 5, 64, vb.BF16, 0)]
        assert vy == [(y.data_ptr(), 3 * 5 * 64, 5 * 64, 64, 2, 3, 5, 64, vb.F32, 0)]
        vb.vsa2_rope_apply(rope, x, y, positions=pos)
        assert seen["rope"][1] == [(0, 0, 0, 0, pos.data_ptr(), 15)] and seen["rope"][5] == 77
        one = FakeTensor(torch.zeros(5, 3, dtype=torch.int32))
        vb.vsa2_rope_apply(rope, x, y, positions=one)
        assert seen["rope"][1] == [(0, 0, 0, 0, one.data_ptr(), 0)]
        for bad in (torch.zeros(2, 4, 3, dtype=torch.int32), torch.zeros(3, 5, 3, dtype=torch.int32), torch.zeros(2, 5, 3, dtype=torch.int64),
                    torch.zeros(2, 3, 5, dtype=torch.int32).transpose(1, 2)):
            with pytest.raises(ValueError):
                vb.vsa2_rope_apply(rope, x, y, positions=FakeTensor(bad))
        w = [FakeTensor(torch.zeros(64)) for _ in range(4)]
        vb.vsa2_qkv_fwd(None, (x, None, x), [y, None, y], w[0], None, eps=0.25, grid=[1, 1, 5])
        r, p, n, vx, vy, _ = seen["fwd"]
        assert r is None and n == [(w[0].data_ptr(), None, 0.25, 0)] and p == [(1, 1, 5, 0, None, 0)]
        assert vx[1] == (None, 0, 0, 0, 2, 0, 5, 64, vb.BF16, 0) and vx[0] == vx[2] and vy[1][5] == 0 and vy[1][8] == vb.F32
        vb.vsa2_qkv_fwd(rope, (x, x, x), (y, y, y), norm=False, grid=(1, 1, 5))
        assert seen["fwd"][2] is None
        for bad in (torch.zeros(63), torch.zeros(64, dtype=torch.float64), torch.zeros(128)[::2]):
            with pytest.raises(ValueError):
                vb.vsa2_qkv_fwd(rope, (x, x, x), (y, y, y), FakeTensor(bad), grid=(1, 1, 5))
        ws = FakeTensor(torch.zeros(100, dtype=torch.float32))
        vb.vsa2_qkv_bwd(rope, (x, x, None), (y, y, y), (x, x, x), w[0], w[1], w[2], None, ws, grid=(1, 1, 5))
        a = seen["bwd"]
        assert a[6:9] == [w[2].data_ptr(), None, ws.data_ptr()] and a[9] == 400 and len(a[3]) == 2 and a[4][0][0] == y.data_ptr()
        vb.vsa2_qkv_bwd(rope, None, (y, y, y), (x, x, x), None, None, None, None, None, norm=False, grid=(1, 1, 5))
        assert seen["bwd"][2] is None and seen["bwd"][3] is None and seen["bwd"][9] == 0
        f8 = lambda rows, cols: vb.Fp8(FakeTensor(torch.zeros(rows, -(-cols // 16) * 16).to(torch.float8_e4m3fn)[:, :cols]),
                                       FakeTensor(torch.zeros(-(-cols // 512), rows, 4, dtype=torch.uint8)))
        mat, out, out_t = FakeTensor(torch.zeros(6, 50)[:, :40]), f8(6, 40), f8(40, 6)
        vb.vsa2_fp8_quantize(mat, out, out_t, squares=True)
        a = seen["qz"]
        assert a[:6] == [mat.data_ptr(), vb.F32, 6, 40, 50, 1] and a[6] == [(out.values.data_ptr(), out.scales.data_ptr(), 48)]
        assert a[7] == [(out_t.values.data_ptr(), out_t.scales.data_ptr(), 16)]
        for bad in ((mat, out_t), (mat, None, out)):
            with pytest.raises(ValueError):
                vb.vsa2_fp8_quantize(*bad)
        c = FakeTensor(torch.zeros(6, 9, dtype=torch.bfloat16)[:, :7])
        vb.vsa2_fp8_matmul(f8(6, 40), f8(7, 40), c, ws)
        a = seen["mm"]
        assert a[:3] == [6, 7, 40] and a[5:10] == [c.data_ptr(), vb.BF16, 9, ws.data_ptr(), 400]
        for bad in ((f8(6, 40), f8(7, 39), c), (f8(5, 40), f8(7, 40), c), (f8(6, 40), f8(8, 40), c)):
            with pytest.raises(ValueError):
                vb.vsa2_fp8_matmul(*bad, ws)
        with pytest.raises(ValueError):
            vb.vsa2_fp8_matmul(f8(6, 40), f8(7, 40), FakeTensor(torch.zeros(6, 7, dtype=torch.float16)), ws)
    finally:
        m.bind(types, real, vb._stream)


def test_marshalling_leaks_no_references():
    import gc
    import sys
    rope, t = vb.vsa2_rope_plan(64, (16, 24, 24)), torch.zeros(1, 1, 4, 64)
    grid, f = (1, 1, 4), vb.Fp8.empty(4, 20, device="cpu")
    objects = (rope, t, grid, f, f.values, f.scales, torch.float32, vb._stream)
    counts = [sys.getrefcount(o) for o in objects]
    for _ in range(200):
        for call in (lambda: vb.vsa2_rope_apply(rope, t, t, grid=grid), lambda: vb.vsa2_qkv_fwd(rope, (t, None, t), (t, t, t), grid=grid),
                     lambda: vb.vsa2_fp8_quantize(t[0, 0], f), lambda: vb.vsa2_fp8_matmul(f, f, t[0, 0], t)):
            with pytest.raises(ValueError):
                call()
        vb.Fp8(f.values, f.scales)
    gc.collect()
    assert all(abs(sys.getrefcount(o) - c) <= 2 for o, c in zip(objects, counts))
