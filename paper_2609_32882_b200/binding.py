"""Binding of libvsa2.so: argument marshalling only (ctypes, and for the short calls csrc/marshal.c), every step runs in the CUDA library.

The functions ``vsa2_query_sizes``, ``vsa2_route``, ``vsa2_attn_fwd``, ``vsa2_attn_bwd`` and
``vsa2_device_status`` mirror the C entry points of ``include/vsa2.h`` and take torch CUDA tensors
(used only for their device pointers) or raw integer addresses.  ``Vsa2Attention`` is a
convenience wrapper that allocates the outputs, maps and workspaces with torch and calls
them in order.  There is no fallback: if the library cannot be loaded, or a call returns an
error code, a ``Vsa2Error`` is raised.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libvsa2.so")

PER_SEQUENCE, PER_QUERY, PER_QUERY_BUDGET = 0, 1, 2
BF16, F32 = 0, 1
FLAG_NO_COARSE = 1
FLAG_EXACT_MAX_FWD = 2
FLAG_FAST_BWD = 4
FLAG_PRECISE_BWD = 8
FLAG_BF16_COARSE_FWD = 64
FLAG_GROUP_ROUTING = 256
FLAG_SELECT_NO_CLUSTERS = 512
ROPE_PAIRS, ROPE_HALVES = 0, 1

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_MISALIGNED = -1, -2, -3, -4
ERR_CUDA, ERR_DEVICE_TIMEOUT, ERR_MAP_OVERFLOW = -5, -6, -7
ERR_STATIC_SCRATCH = -8

EXPORTS = ("vsa2_query_sizes", "vsa2_route", "vsa2_route_scores", "vsa2_attn_fwd", "vsa2_attn_bwd",
           "vsa2_device_status", "vsa2_strerror", "vsa2_profile_events", "vsa2_launch_count", "vsa2_selftest_umma", "vsa2_route_noalloc", "vsa2_last_cuda_error",
           "vsa2_gate_fwd", "vsa2_gate_bwd", "vsa2_gate_bwd_add", "vsa2_gate_bwd_workspace_bytes",
           "vsa2_attn_bwd_preferred_workspace_bytes", "vsa2_attn_bwd_scratch", "vsa2_attn_bwd_scratch_bytes",
           "vsa2_route_scratch", "vsa2_route_scratch_bytes", "vsa2_permute_cube_major",
           "vsa2_selftest_timeout", "vsa2_debug_rescue_capacity", "vsa2_selftest_divmod",
           "vsa2_rope_plan", "vsa2_rope_apply", "vsa2_qkv_fwd", "vsa2_qkv_bwd", "vsa2_qkv_bwd_workspace_bytes",
           "vsa2_fp8_quantize", "vsa2_fp8_matmul", "vsa2_fp8_matmul_workspace_bytes", "vsa2_debug_fp8_matmul_plan",
           "vsa2_residual_norm_fwd", "vsa2_residual_norm_bwd", "vsa2_residual_norm_bwd_workspace_bytes", "vsa2_dropout",
           "vsa2_int8_quantize", "vsa2_int8_matmul", "vsa2_int8_matmul_workspace_bytes", "vsa2_debug_int8_matmul_plan",
           "vsa2_debug_residual_norm_rows")

KERNELS = ("pool", "router_lse", "router_pool", "select", "coarse_fwd", "fine_fwd", "bwd_pre", "coarse_bwd",
           "fine_bwd_dq", "fine_bwd_dkv", "pool_router")


class Vsa2Error(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        msg = _lib().vsa2_strerror(code).decode() if _LIB is not None else "library not loaded"
        if code == ERR_CUDA and _LIB is not None:
            msg += ": " + _lib().vsa2_last_cuda_error().decode()
        super().__init__(f"{where}: {msg} (code {code})")


class Params(C.Structure):
    _fields_ = [("batch", C.c_int32), ("heads_q", C.c_int32), ("heads_kv", C.c_int32), ("head_dim", C.c_int32),
                ("grid_t", C.c_int32), ("grid_h", C.c_int32), ("grid_w", C.c_int32),
                ("cube_t", C.c_int32), ("cube_h", C.c_int32), ("cube_w", C.c_int32),
                ("rpool_t", C.c_int32), ("rpool_h", C.c_int32), ("rpool_w", C.c_int32),
                ("select_mode", C.c_int32), ("topk", C.c_int32), ("keep_fraction", C.c_float),
                ("softmax_scale", C.c_float), ("out_dtype", C.c_int32), ("flags", C.c_int32), ("text_len", C.c_int32),
                ("nnz_cap", C.c_int64)]


class Sizes(C.Structure):
    _fields_ = [("n_cubes", C.c_int32), ("n_subcubes", C.c_int32), ("block_tokens", C.c_int32),
                ("topk_eff", C.c_int32), ("seq_len", C.c_int64), ("nnz_cap", C.c_int64),
                ("ptr_elems", C.c_int64), ("idx_elems", C.c_int64), ("pooled_q_elems", C.c_int64),
                ("pooled_kv_elems", C.c_int64), ("lse_c_elems", C.c_int64), ("o_res_elems", C.c_int64),
                ("route_workspace_bytes", C.c_size_t), ("fwd_workspace_bytes", C.c_size_t),
                ("bwd_workspace_bytes", C.c_size_t), ("tokens_per_head", C.c_int64), ("text_blocks", C.c_int32),
                ("reserved", C.c_int32)]


class Map(C.Structure):
    _fields_ = [("row_ptr", C.c_void_p), ("col_idx", C.c_void_p), ("col_ptr", C.c_void_p), ("row_idx", C.c_void_p)]


class Saved(C.Structure):
    _fields_ = [("qc", C.c_void_p), ("kc", C.c_void_p), ("vc", C.c_void_p), ("oc_hat", C.c_void_p),
                ("lse_c", C.c_void_p), ("o_res", C.c_void_p)]


class Rope(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("layout", C.c_int32), ("axis_pairs", C.c_int32 * 3), ("reserved", C.c_int32),
                ("turn", C.c_uint64 * 64)]


# (the structs below: for callers of the library's functions themselves; the wrappers go through csrc/marshal.c)
class Place(C.Structure):
    _fields_ = [("grid_t", C.c_int32), ("grid_h", C.c_int32), ("grid_w", C.c_int32), ("first", C.c_int32),
                ("positions", C.c_void_p), ("positions_batch_stride", C.c_int64)]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("head_stride", C.c_int64), ("token_stride", C.c_int64),
                ("batch", C.c_int32), ("heads", C.c_int32), ("tokens", C.c_int32), ("channels", C.c_int32),
                ("dtype", C.c_int32), ("reserved", C.c_int32)]


class QkNorm(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("eps", C.c_float), ("reserved", C.c_int32)]


class Fp8Matrix(C.Structure):
    _fields_ = [("values", C.c_void_p), ("scales", C.c_void_p), ("ld", C.c_int64)]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("ld", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class Drop(C.Structure):
    _fields_ = [("rng", C.c_void_p), ("p", C.c_double)]


class Int8Matrix(C.Structure):
    _fields_ = [("values", C.c_void_p), ("scales", C.c_void_p), ("ld", C.c_int64)]


_LIB = None


def _lib():
    """Loads libvsa2.so (built in-tree by ``build.build_library``); raises if it is missing."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2609_32882_b200.build` (nvcc, sm_100a)")
        lib = C.CDLL(LIB_PATH)
        vp, sz, i32p = C.c_void_p, C.c_size_t, C.POINTER(C.c_int32)
        lib.vsa2_query_sizes.argtypes = [C.POINTER(Params), C.POINTER(Sizes)]
        lib.vsa2_route.argtypes = [C.POINTER(Params), vp, vp, vp, C.POINTER(Map), vp, sz, vp]
        lib.vsa2_route_scratch.argtypes = lib.vsa2_route.argtypes[:-1] + [vp, sz, vp]
        lib.vsa2_route_noalloc.argtypes = [C.POINTER(Params), vp, vp, vp, C.POINTER(Map), vp, vp]
        lib.vsa2_permute_cube_major.argtypes = [C.POINTER(Params), C.c_int32, C.c_int32, vp, vp, vp]
        lib.vsa2_gate_fwd.argtypes = [C.POINTER(Params), C.c_int32, vp, vp, vp, vp]
        for fn in (lib.vsa2_attn_bwd_preferred_workspace_bytes, lib.vsa2_attn_bwd_scratch_bytes, lib.vsa2_route_scratch_bytes):
            fn.argtypes = [C.POINTER(Params)]
            fn.restype = C.c_size_t
        lib.vsa2_gate_bwd_workspace_bytes.argtypes = [C.POINTER(Params), C.c_int32]
        lib.vsa2_gate_bwd_workspace_bytes.restype = C.c_size_t
        lib.vsa2_gate_bwd.argtypes = [C.POINTER(Params), C.c_int32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.vsa2_route_scores.argtypes = [C.POINTER(Params), vp]
        lib.vsa2_route_scores.restype = vp
        lib.vsa2_attn_fwd.argtypes = [C.POINTER(Params), vp, vp, vp, vp, C.POINTER(Map), vp, vp, C.POINTER(Saved), vp, sz, vp]
        lib.vsa2_attn_bwd.argtypes = [C.POINTER(Params), vp, vp, vp, vp, C.POINTER(Map), vp, vp, C.POINTER(Saved), vp,
                                      vp, vp, vp, vp, vp, sz, vp]
        lib.vsa2_attn_bwd_scratch.argtypes = lib.vsa2_attn_bwd.argtypes[:-1] + [vp, sz, vp]
        lib.vsa2_device_status.argtypes = [vp, vp, i32p]
        lib.vsa2_last_cuda_error.argtypes = []
        lib.vsa2_last_cuda_error.restype = C.c_char_p
        lib.vsa2_strerror.argtypes = [C.c_int]
        lib.vsa2_strerror.restype = C.c_char_p
        lib.vsa2_profile_events.argtypes = [C.c_int32, vp, vp]
        lib.vsa2_selftest_umma.argtypes = [C.POINTER(Params), vp, vp, vp, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp]
        lib.vsa2_selftest_timeout.argtypes = [C.c_uint32, vp, vp, vp]
        lib.vsa2_debug_rescue_capacity.argtypes = [C.c_int32]
        lib.vsa2_launch_count.argtypes = []
        lib.vsa2_launch_count.restype = C.c_int64
        lib.vsa2_selftest_divmod.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        lib.vsa2_selftest_divmod.restype = C.c_int64
        lib.vsa2_gate_bwd_add.argtypes = [vp, C.c_int32] + [vp] * 6 + [C.c_int64, vp, sz, vp]
        lib.vsa2_rope_plan.argtypes = [C.c_int32, C.c_int32, vp, vp, vp, C.POINTER(Rope)]
        lib.vsa2_rope_apply.argtypes = [vp, vp, vp, vp, C.c_int32, vp]
        lib.vsa2_qkv_fwd.argtypes = [vp] * 6
        lib.vsa2_qkv_bwd.argtypes = [vp] * 9 + [sz, vp]
        lib.vsa2_qkv_bwd_workspace_bytes.argtypes = [C.c_int32]
        lib.vsa2_fp8_quantize.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int32, vp, vp, vp]
        lib.vsa2_fp8_matmul.argtypes = [C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, C.c_int32, C.c_int64, vp, sz, vp]
        lib.vsa2_fp8_matmul_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32]
        lib.vsa2_debug_fp8_matmul_plan.argtypes = [C.c_int32] * 7 + [vp]
        lib.vsa2_residual_norm_fwd.argtypes = [C.c_int32] * 2 + [vp] * 4 + [C.c_float] + [vp] * 5
        lib.vsa2_residual_norm_bwd.argtypes = [C.c_int32] * 2 + [vp] * 5 + [C.c_float] + [vp] * 4 + [sz, vp]
        lib.vsa2_residual_norm_bwd_workspace_bytes.argtypes = [C.c_int32] * 2
        lib.vsa2_dropout.argtypes = [C.c_int32] * 2 + [vp] * 5
        lib.vsa2_int8_quantize.argtypes = [C.c_int32] * 2 + [vp] * 3
        lib.vsa2_int8_matmul.argtypes = [C.c_int32] * 3 + [vp] * 4 + [C.c_int32, C.c_int64, vp, sz, vp]
        lib.vsa2_int8_matmul_workspace_bytes.argtypes = [C.c_int32] * 3
        lib.vsa2_debug_int8_matmul_plan.argtypes = [C.c_int32] * 5 + [vp]
        lib.vsa2_debug_residual_norm_rows.argtypes = [C.c_int32] * 3 + [vp]
        for fn in (lib.vsa2_qkv_bwd_workspace_bytes, lib.vsa2_fp8_matmul_workspace_bytes, lib.vsa2_residual_norm_bwd_workspace_bytes,
                   lib.vsa2_int8_matmul_workspace_bytes):
            fn.restype = C.c_size_t
        for name in EXPORTS:
            if name not in ("vsa2_qkv_bwd_workspace_bytes", "vsa2_fp8_matmul_workspace_bytes", "vsa2_residual_norm_bwd_workspace_bytes",
                            "vsa2_int8_matmul_workspace_bytes",
                            "vsa2_strerror", "vsa2_route_scores", "vsa2_launch_count", "vsa2_last_cuda_error", "vsa2_selftest_divmod",
                            "vsa2_gate_bwd_workspace_bytes", "vsa2_attn_bwd_preferred_workspace_bytes",
                            "vsa2_attn_bwd_scratch_bytes", "vsa2_route_scratch_bytes"):
                getattr(lib, name).restype = C.c_int
        _LIB = lib
    return _LIB


def _ptr(t):
    """Device address of a torch tensor (or an int address, or None)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _current_stream():
    """Handle of the calling thread's current stream, without the Stream object (0.3 us instead of 3.2; a toy grid's calls wait for the host)."""
    import torch
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return raw(device())


def _stream(stream):
    if stream is None:
        return _current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(code, where):
    if code != OK:
        raise Vsa2Error(code, where)


def make_params(batch, heads_q, heads_kv, head_dim, grid, cube=(4, 4, 4), rpool=(2, 2, 2),
                select_mode=PER_SEQUENCE, topk=0, keep_fraction=0.0, softmax_scale=0.0, out_dtype=BF16,
                flags=0, nnz_cap=0, text_len=0) -> Params:
    return Params(batch, heads_q, heads_kv, head_dim, *grid, *cube, *rpool, select_mode, topk, keep_fraction,
                  softmax_scale, out_dtype, flags, text_len, nnz_cap)


def params_from_workload(wl, **overrides) -> Params:
    kw = dict(batch=wl.batch, heads_q=wl.heads_q, heads_kv=wl.heads_kv, head_dim=wl.head_dim, grid=wl.grid,
              cube=wl.cube, rpool=wl.rpool, select_mode=wl.select_mode, topk=wl.topk,
              text_len=getattr(wl, "text_len", 0))
    kw.update(overrides)
    return make_params(**kw)


# ---------------------------------------------------------------------------------------------
# one-to-one wrappers of the C entry points
# ---------------------------------------------------------------------------------------------
def vsa2_query_sizes(p: Params) -> Sizes:
    s = Sizes()
    _check(_lib().vsa2_query_sizes(C.byref(p), C.byref(s)), "vsa2_query_sizes")
    return s


def vsa2_route(p, q, k, budgets, vmap: Map, workspace, workspace_bytes=None, stream=None, scratch=None):
    """`scratch`: None, or a tensor of at least vsa2_route_scratch_bytes(p) bytes (large problems run faster with it)."""
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    args = (C.byref(p), _ptr(q), _ptr(k), _ptr(budgets), C.byref(vmap), _ptr(workspace), nbytes)
    if scratch is None:
        _check(_lib().vsa2_route(*args, _stream(stream)), "vsa2_route")
    else:
        _check(_lib().vsa2_route_scratch(*args, _ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)),
               "vsa2_route_scratch")


def vsa2_route_scratch_bytes(p) -> int:
    """Bytes of scratch with which the router runs fastest (0: it has no use for any)."""
    return int(_lib().vsa2_route_scratch_bytes(C.byref(p)))


def vsa2_route_noalloc(p, q, k, budgets, vmap: Map, device_status=None, stream=None):
    """Router + selection without a caller workspace (scratch is a fixed 8 MiB array inside the library).

    For callers that cannot allocate device memory at this point; problems needing more scratch raise
    Vsa2Error(ERR_STATIC_SCRATCH).  `device_status`: optional int32 CUDA tensor receiving the status word."""
    _check(_lib().vsa2_route_noalloc(C.byref(p), _ptr(q), _ptr(k), _ptr(budgets), C.byref(vmap), _ptr(device_status),
                                     _stream(stream)), "vsa2_route_noalloc")


def vsa2_permute_cube_major(p, heads, src, dst, inverse=False, stream=None):
    """Raster [B, heads, L, D] -> cube-major [B, heads, N*B, D] (zero padding), or back with inverse=True; bf16."""
    _check(_lib().vsa2_permute_cube_major(C.byref(p), heads, 1 if inverse else 0, _ptr(src), _ptr(dst), _stream(stream)),
           "vsa2_permute_cube_major")


def vsa2_gate_fwd(p, hidden, x, w_g, gate, stream=None):
    """gate[b, h, l] = tanh(sum_c x[b, l, c] w_g[c, h]) (Eq. 13); x [B, L, hidden] bf16, w_g [hidden, Hq] bf16, gate [B, Hq, L] fp32."""
    _check(_lib().vsa2_gate_fwd(C.byref(p), hidden, _ptr(x), _ptr(w_g), _ptr(gate), _stream(stream)), "vsa2_gate_fwd")


def vsa2_gate_bwd_workspace_bytes(p, hidden) -> int:
    return int(_lib().vsa2_gate_bwd_workspace_bytes(C.byref(p), hidden))


def vsa2_gate_bwd(p, hidden, x, w_g, gate, dgate, d_w_g, dx, workspace, stream=None):
    """Backward of vsa2_gate_fwd: d_w_g [hidden, Hq] fp32 and dx [B, L, hidden] (the params' output dtype)."""
    nbytes = workspace.numel() * workspace.element_size()
    _check(_lib().vsa2_gate_bwd(C.byref(p), hidden, _ptr(x), _ptr(w_g), _ptr(gate), _ptr(dgate), _ptr(d_w_g), _ptr(dx),
                                _ptr(workspace), nbytes, _stream(stream)), "vsa2_gate_bwd")


def vsa2_gate_bwd_add(p, hidden, x, w_g, gate, dgate, d_w_g, dx, workspace, stream=None):
    """vsa2_gate_bwd with its dx added to what `dx` holds: [B, L or more rows, hidden], contiguous but for its batch entries' distance; rows from L on stay."""
    import torch
    video, dtype, shape, strides = p.grid_t * p.grid_h * p.grid_w, torch.float32 if p.out_dtype == F32 else torch.bfloat16, dx.shape, dx.stride()
    if not (len(shape) == 3 and shape[0] == p.batch and shape[1] >= video and shape[2] == hidden and (shape[1] == 1 or strides[1] == hidden) and strides[2] == 1 and
            dx.is_cuda and dx.dtype == dtype):
        raise ValueError(f"expected dx as a CUDA tensor [{p.batch}, {video} or more, {hidden}] in {dtype} with contiguous batch entries")
    nbytes = workspace.numel() * workspace.element_size()
    _check(_lib().vsa2_gate_bwd_add(C.byref(p), hidden, _ptr(x), _ptr(w_g), _ptr(gate), _ptr(dgate), _ptr(d_w_g), dx.data_ptr(), strides[0], _ptr(workspace),
                                    nbytes, _stream(stream)), "vsa2_gate_bwd_add")


def vsa2_route_scores(p, workspace) -> int:
    return _lib().vsa2_route_scores(C.byref(p), _ptr(workspace))


def vsa2_attn_fwd(p, q, k, v, gate, vmap: Map, o, lse, saved, workspace, workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(_lib().vsa2_attn_fwd(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(gate), C.byref(vmap), _ptr(o), _ptr(lse),
                                C.byref(saved) if saved is not None else None, _ptr(workspace), nbytes,
                                _stream(stream)), "vsa2_attn_fwd")


def vsa2_attn_bwd(p, q, k, v, gate, vmap: Map, o, lse, saved, d_o, dq, dk, dv, dgate, workspace,
                  workspace_bytes=None, stream=None, scratch=None):
    """`scratch`: None (what `workspace` holds beyond the least serves as scratch) or a tensor of its own."""
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    args = (C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(gate), C.byref(vmap), _ptr(o), _ptr(lse),
            C.byref(saved) if saved is not None else None, _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dgate), _ptr(workspace), nbytes)
    if scratch is None:
        _check(_lib().vsa2_attn_bwd(*args, _stream(stream)), "vsa2_attn_bwd")
    else:
        _check(_lib().vsa2_attn_bwd_scratch(*args, _ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)),
               "vsa2_attn_bwd_scratch")


def vsa2_attn_bwd_scratch_bytes(p) -> int:
    """Bytes of scratch with which the backward runs fastest (0: it has no use for any)."""
    return int(_lib().vsa2_attn_bwd_scratch_bytes(C.byref(p)))


def vsa2_attn_bwd_preferred_workspace_bytes(p) -> int:
    """Bytes of backward workspace with which vsa2_attn_bwd runs fastest (at least sizes.bwd_workspace_bytes)."""
    return int(_lib().vsa2_attn_bwd_preferred_workspace_bytes(C.byref(p)))


# ---------------------------------------------------------------------------------------------
# between a layer's hidden states and its attention
# ---------------------------------------------------------------------------------------------
def vsa2_rope_plan(head_dim, channels, theta=1e4, scale=1.0, layout=ROPE_PAIRS) -> Rope:
    """Rotary positions on (t, h, w): `channels` of a head turn with each axis, pair j of axis a by scale theta^(-2 j / channels[a])
    radians per position.  theta, scale: one number, or one for each axis."""
    three = lambda v: (v, v, v) if isinstance(v, (int, float)) else tuple(v)
    theta, scale, channels = three(theta), three(scale), tuple(channels)
    if not len(theta) == len(scale) == len(channels) == 3:
        raise ValueError("three axes are expected: (t, h, w)")
    out = Rope()
    _check(_lib().vsa2_rope_plan(head_dim, layout, (C.c_int32 * 3)(*channels), (C.c_double * 3)(*theta), (C.c_double * 3)(*scale),
                                 C.byref(out)), "vsa2_rope_plan")
    return out


# These calls are marshalled by a small module of C (csrc/marshal.c): a toy grid's calls wait for the host.
MARSHAL_PATH = os.path.join(HERE, "_marshal.so")
_MARSHAL = None


def _marshal():
    """The module (built in-tree with the library); raises if it is missing."""
    global _MARSHAL
    if _MARSHAL is None:
        import importlib.machinery
        import importlib.util

        import torch
        if not os.path.exists(MARSHAL_PATH):
            raise FileNotFoundError(f"{MARSHAL_PATH} not found: build it with `python -m paper_2609_32882_b200.build`")
        loader = importlib.machinery.ExtensionFileLoader("_marshal", MARSHAL_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_marshal", MARSHAL_PATH, loader=loader))
        loader.exec_module(module)
        lib = _lib()
        at = lambda *functions: tuple(C.cast(f, C.c_void_p).value for f in functions)
        module.bind((torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn, torch.uint8),
                    at(lib.vsa2_rope_apply, lib.vsa2_qkv_fwd, lib.vsa2_qkv_bwd, lib.vsa2_fp8_quantize, lib.vsa2_fp8_matmul), _stream)
        module.bind_rows((torch.int8, torch.int64), at(lib.vsa2_residual_norm_fwd, lib.vsa2_residual_norm_bwd, lib.vsa2_dropout, lib.vsa2_int8_quantize,
                                                       lib.vsa2_int8_matmul),
                         getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device, getattr(torch._C, "_cuda_getCurrentRawStream", None))
        _MARSHAL = module
    return _MARSHAL


def vsa2_rope_apply(rope, x, y, grid=None, first=0, positions=None, inverse=False, stream=None):
    """y = R(position) x, or with `inverse` its inverse (the gradient); tensors [batch, heads, tokens, D], bf16 or fp32, any strides; y may be x.
    Positions: rows first, first + 1, .. of the raster of `grid` (rows behind it do not turn), or int32 [batch or 1, tokens, 3]."""
    code = (_MARSHAL or _marshal()).rope_apply(rope, x, y, grid, first, positions, inverse, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_rope_apply")


def vsa2_qkv_fwd(rope, x, y, q_weight=None, k_weight=None, eps=1e-6, norm=True, grid=None, first=0, positions=None, stream=None):
    """x = (q, k, v) as the projection leaves them -> y = (q, k, v) of the attention: norm of every head of q and k, weights, rotation (rope None:
    none), v copied.  All are [batch, heads, tokens, D] views of any strides; a member may be None on both sides."""
    code = (_MARSHAL or _marshal()).qkv_fwd(rope, x, y, q_weight, k_weight, eps, norm, grid, first, positions, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_qkv_fwd")


def vsa2_qkv_bwd_workspace_bytes(channels) -> int:
    return int(_lib().vsa2_qkv_bwd_workspace_bytes(channels))


def vsa2_qkv_bwd(rope, x, dy, dx, q_weight, k_weight, d_q_weight, d_k_weight, workspace, eps=1e-6, norm=True, grid=None, first=0,
                 positions=None, stream=None):
    """Backward of vsa2_qkv_fwd: x = its inputs (q, k and, unused, v), dy = gradients of its outputs -> dx, and the weights' gradients (fp32, None: not
    wanted).  workspace: vsa2_qkv_bwd_workspace_bytes(D) bytes (None without a norm)."""
    code = (_MARSHAL or _marshal()).qkv_bwd(rope, x, dy, dx, q_weight, k_weight, d_q_weight, d_k_weight, workspace, eps, norm, grid, first, positions,
                                            stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_qkv_bwd")


class Fp8:
    """A matrix [rows, cols] in 8-bit form: `values` float8_e4m3fn [rows, cols] whose rows begin on 16-byte boundaries, `scales` uint8
    [ceil(cols / 512), rows, 4] (exponents + 127, one for each 128 values of a row)."""
    __slots__ = ("values", "scales")

    def __init__(self, values, scales):
        (_MARSHAL or _marshal()).check_fp8(values, scales)
        self.values, self.scales = values, scales

    @classmethod
    def empty(cls, rows, cols, device="cuda"):
        import torch
        room = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.float8_e4m3fn, device=device)
        return cls(room[:, :cols], torch.empty(-(-cols // 512), rows, 4, dtype=torch.uint8, device=device))

    @property
    def shape(self):
        return tuple(self.values.shape)

    def dequantize(self):
        """The matrix in fp32 (torch operations: for inspection and tests)."""
        import torch
        rows, cols = self.values.shape
        e = self.scales.transpose(0, 1).reshape(rows, 4 * self.scales.shape[0]).to(torch.int32) - 127
        return self.values.float() * torch.ldexp(torch.ones(e.shape, device=e.device), e).repeat_interleave(128, dim=1)[:, :cols]


def vsa2_fp8_quantize(x, out=None, out_t=None, squares=False, stream=None):
    """x [rows, cols] (bf16 or fp32, contiguous rows) -> `out`, its 8-bit form, and / or `out_t`, that of its transpose.  squares: one scale for each
    128 x 128 values instead of each 128 of a row."""
    code = (_MARSHAL or _marshal()).quantize(x, out, out_t, squares, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_fp8_quantize")


def vsa2_fp8_matmul_workspace_bytes(m, n, k) -> int:
    return int(_lib().vsa2_fp8_matmul_workspace_bytes(m, n, k))


def fp8_matmul_workspace(m, n, k, device="cuda"):
    """Workspace of vsa2_fp8_matmul for products up to this size that follow one another on a stream."""
    import torch
    workspace = torch.empty(vsa2_fp8_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=device)
    workspace[:256].zero_()          # status block
    return workspace


def vsa2_fp8_matmul(a, b, c, workspace, stream=None):
    """c [m, n] = a b^T of two Fp8 matrices [m, k] and [n, k]; c bf16 or fp32 with contiguous rows."""
    code = (_MARSHAL or _marshal()).matmul(a, b, c, workspace, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_fp8_matmul")


def vsa2_debug_fp8_matmul_plan(m, n, k, c_dtype=BF16, c_aligned=True, sms=148, pairs=True):
    """(columns of a tile, CTAs that share one, whether A's rows are its lanes, ranges of K, tiles along the columns' operand, tiles taken together); host arithmetic."""
    out = (C.c_int32 * 6)()
    _check(_lib().vsa2_debug_fp8_matmul_plan(m, n, k, c_dtype, c_aligned, sms, pairs, out), "vsa2_debug_fp8_matmul_plan")
    return tuple(out)


# ---------------------------------------------------------------------------------------------
# the residual stream around a layer
# ---------------------------------------------------------------------------------------------
class Int8:
    """A matrix [rows, cols] in 8-bit whole numbers: `values` int8 [rows, cols] whose rows begin on 16-byte boundaries, `scales` fp32 [rows]."""
    __slots__ = ("values", "scales")

    def __init__(self, values, scales):
        (_MARSHAL or _marshal()).check_int8(values, scales)
        self.values, self.scales = values, scales

    @classmethod
    def empty(cls, rows, cols, device="cuda"):
        import torch
        room = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device=device)
        return cls(room[:, :cols], torch.empty(rows, dtype=torch.float32, device=device))

    @property
    def shape(self):
        return tuple(self.values.shape)

    def dequantize(self):
        """The matrix in fp32 (torch operations: for inspection and tests)."""
        return self.values.float() * self.scales.unsqueeze(1)


def vsa2_residual_norm_fwd(x, residual=None, weight=None, eps=1e-6, h=None, y=None, y_fp8=None, y_int8=None, p=0.0, rng=None, stream=None):
    """h = residual + dropout(x), y = h / sqrt(mean over the row of h^2 + eps) * weight, of matrices [rows, cols] (bf16 or fp32, contiguous rows).  Written are the
    outputs that are given: h (of the residual's type, without one of x's), y (bf16 or fp32), y_fp8 (Fp8), y_int8 (Int8).  h may be x or residual itself.  weight: fp32 [cols], None:
    ones.  p, rng: as vsa2_dropout."""
    code = (_MARSHAL or _marshal()).norm_fwd(x, residual, weight, eps, h, y, y_fp8, y_int8, p, rng, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_residual_norm_fwd")


def vsa2_residual_norm_bwd_workspace_bytes(rows, cols) -> int:
    return int(_lib().vsa2_residual_norm_bwd_workspace_bytes(rows, cols))


def vsa2_residual_norm_bwd(h, dy, dh=None, weight=None, eps=1e-6, d_residual=None, dx=None, d_weight=None, workspace=None, p=0.0, rng=None, stream=None):
    """Backward of vsa2_residual_norm_fwd: h, the gradient dy of y and dh of h (None: none; of h's type) -> what is given of d_residual (h's type), dx (through the dropout; without
    one, and in h's type, d_residual is x's gradient too) and d_weight (fp32 [cols]).  workspace: vsa2_residual_norm_bwd_workspace_bytes(rows, cols) bytes (None without d_weight)."""
    code = (_MARSHAL or _marshal()).norm_bwd(h, dy, dh, weight, eps, d_residual, dx, d_weight, workspace, p, rng, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_residual_norm_bwd")


def vsa2_dropout(x, y, p, rng, residual=None, stream=None):
    """y = x / (1 - p) where an element is kept, else zero, plus the residual (of y's type) where one is given; y may be x or residual itself.  The mask follows from rng (int64 [2] on the
    device: seed, offset) and an element's place; the backward is the same call on the gradient.  rng is read when the kernel runs: a captured graph draws anew when it changes."""
    code = (_MARSHAL or _marshal()).dropout(x, y, p, rng, residual, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_dropout")


def vsa2_int8_quantize(x, out, stream=None):
    """x [rows, cols] (bf16 or fp32, contiguous rows) -> `out` (Int8): each row's values times 127 over its largest magnitude, rounded to nearest."""
    code = (_MARSHAL or _marshal()).int8_quantize(x, out, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_int8_quantize")


def vsa2_int8_matmul_workspace_bytes(m, n, k) -> int:
    return int(_lib().vsa2_int8_matmul_workspace_bytes(m, n, k))


def int8_matmul_workspace(m, n, k, device="cuda"):
    """Workspace of vsa2_int8_matmul for products up to this size that follow one another on a stream."""
    import torch
    workspace = torch.empty(vsa2_int8_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device=device)
    workspace[:256].zero_()          # status block
    return workspace


def vsa2_int8_matmul(a, b, c, workspace, bias=None, stream=None):
    """c [m, n] = a b^T of two Int8 matrices [m, k] and [n, k], plus bias (fp32 [n]); c bf16 or fp32 with contiguous rows."""
    code = (_MARSHAL or _marshal()).int8_matmul(a, b, c, workspace, bias, stream)
    if code != OK:
        raise Vsa2Error(code, "vsa2_int8_matmul")


def vsa2_debug_int8_matmul_plan(m, n, k, sms=148, pairs=True):
    """(columns of a tile, 8: the kernel of few rows of a; CTAs that share one; ranges of K; tiles along a, and those taken together); host arithmetic."""
    out = (C.c_int32 * 5)()
    _check(_lib().vsa2_debug_int8_matmul_plan(m, n, k, sms, pairs, out), "vsa2_debug_int8_matmul_plan")
    return tuple(out)


def vsa2_debug_residual_norm_rows(rows, resident, cta):
    """(CTAs of vsa2_residual_norm_fwd and vsa2_int8_quantize on a device that holds `resident`, rows of CTA `cta`, the last of them); host arithmetic."""
    out = (C.c_int64 * 3)()
    _check(_lib().vsa2_debug_residual_norm_rows(rows, resident, cta, out), "vsa2_debug_residual_norm_rows")
    return tuple(out)


def vsa2_profile_events(kernel_id: int, start_event, stop_event):
    """start/stop: torch.cuda.Event objects (already recorded once, so that their handles exist) or None."""
    a = None if start_event is None else start_event.cuda_event
    b = None if stop_event is None else stop_event.cuda_event
    _check(_lib().vsa2_profile_events(kernel_id, a, b), "vsa2_profile_events")


def vsa2_selftest_umma(p, q, k, v, cube_q, cube_a, cube_b, p_t, s_t_out, o_t_out, k_tile_dump, status, stream=None):
    _check(_lib().vsa2_selftest_umma(C.byref(p), _ptr(q), _ptr(k), _ptr(v), cube_q, cube_a, cube_b, _ptr(p_t),
                                     _ptr(s_t_out), _ptr(o_t_out), _ptr(k_tile_dump), _ptr(status), _stream(stream)),
           "vsa2_selftest_umma")


def vsa2_launch_count() -> int:
    return int(_lib().vsa2_launch_count())


def vsa2_device_status(workspace, stream=None) -> int:
    out = C.c_int32(0)
    _check(_lib().vsa2_device_status(_ptr(workspace), _stream(stream), C.byref(out)), "vsa2_device_status")
    return out.value


# ---------------------------------------------------------------------------------------------
# convenience wrapper: owns maps, saved state and workspaces (torch is used for memory only)
# ---------------------------------------------------------------------------------------------
class Vsa2Attention:
    """Allocates what the C ABI wants with torch and calls route / forward / backward."""

    def __init__(self, params: Params, device="cuda"):
        import torch
        self.torch = torch
        self.p = params
        self.sizes = vsa2_query_sizes(params)
        s = self.sizes
        dev = torch.device(device)
        i32 = dict(dtype=torch.int32, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        self.row_ptr = torch.empty(s.ptr_elems, **i32)
        self.col_idx = torch.empty(max(1, s.idx_elems), **i32)
        self.col_ptr = torch.empty(s.ptr_elems, **i32)
        self.row_idx = torch.empty(max(1, s.idx_elems), **i32)
        self.map = Map(self.row_ptr.data_ptr(), self.col_idx.data_ptr(), self.col_ptr.data_ptr(), self.row_idx.data_ptr())
        self.qc = torch.empty(s.pooled_q_elems, **f32)
        self.kc = torch.empty(s.pooled_kv_elems, **f32)
        self.vc = torch.empty(s.pooled_kv_elems, **f32)
        self.oc_hat = torch.empty(s.pooled_q_elems, **f32)
        self.lse_c = torch.empty(s.lse_c_elems, **f32)
        self.o_res = torch.empty(s.o_res_elems, dtype=torch.bfloat16, device=dev) if s.o_res_elems else None
        self.saved = Saved(self.qc.data_ptr(), self.kc.data_ptr(), self.vc.data_ptr(), self.oc_hat.data_ptr(),
                           self.lse_c.data_ptr(), self.o_res.data_ptr() if s.o_res_elems else None)
        u8 = dict(dtype=torch.uint8, device=dev)
        self.ws_route = torch.empty(s.route_workspace_bytes, **u8)
        self.ws_fwd = torch.empty(s.fwd_workspace_bytes, **u8)
        # scratch of a route call (large problems: 0.05 - 0.3 GB), like the one below
        self.route_scratch_bytes = vsa2_route_scratch_bytes(params)
        # scratch of a backward call, up to 8 GiB: taken from torch's allocator for the call and given back, so the handles of a
        # model share it and one that only runs forward has none; 0 = none (the dQ pass recomputes the score gradients).  Up to
        # 1 MiB (a toy grid, whose passes wait for the host) is part of the workspace instead: asking takes 3 us
        self.bwd_scratch_bytes = vsa2_attn_bwd_scratch_bytes(params)
        if self.bwd_scratch_bytes <= 1 << 20:
            self.bwd_scratch_bytes = 0
            self.ws_bwd = torch.empty(vsa2_attn_bwd_preferred_workspace_bytes(params), **u8)
        else:
            self.ws_bwd = torch.empty(s.bwd_workspace_bytes, **u8)
        for ws in (self.ws_route, self.ws_fwd, self.ws_bwd):
            ws[:256].zero_()          # status block
        self._refused = {}            # scratch there was no room for: {attribute: [bytes, calls it is done without, calls left]}
        self.out_torch_dtype = torch.float32 if params.out_dtype == F32 else torch.bfloat16

    # shapes ---------------------------------------------------------------------------------
    def map_views(self):
        """(row_ptr [B,Hq,N+1], col_idx [B,Hq,nnz_cap], col_ptr, row_idx) as torch views."""
        p, s = self.p, self.sizes
        shp = (p.batch, p.heads_q)
        return (self.row_ptr.view(*shp, s.n_cubes + 1), self.col_idx[:s.idx_elems].view(*shp, s.nnz_cap),
                self.col_ptr.view(*shp, s.n_cubes + 1), self.row_idx[:s.idx_elems].view(*shp, s.nnz_cap))

    def scores(self):
        """P_r [B,Hq,N,N] fp32 left in the route workspace by the last route() call (a copy)."""
        p, s = self.p, self.sizes
        addr = vsa2_route_scores(p, self.ws_route)
        off = addr - self.ws_route.data_ptr()
        n = p.batch * p.heads_q * s.n_cubes * s.n_cubes
        return self.ws_route[off:off + 4 * n].view(self.torch.float32).view(p.batch, p.heads_q, s.n_cubes, s.n_cubes).clone()

    # calls ----------------------------------------------------------------------------------
    def route(self, q, k, budgets=None, stream=None):
        vsa2_route(self.p, q, k, budgets, self.map, self.ws_route, stream=stream,
                   scratch=self._scratch("route_scratch_bytes", q.device, stream))

    def forward(self, q, k, v, gate, o=None, lse=None, stream=None):
        p = self.p
        if o is None:
            o = self._empty_like(q, q.device)
        if lse is None:
            lse = self._empty_f32(q, q.shape[:-1])
        vsa2_attn_fwd(p, q, k, v, gate, self.map, o, lse, self.saved, self.ws_fwd, stream=stream)
        return o, lse

    def backward(self, q, k, v, gate, o, lse, d_o, dq=None, dk=None, dv=None, dgate=None, stream=None):
        p = self.p
        if dq is None:
            dq = self._empty_like(q, q.device)
        if dk is None:
            dk = self._empty_like(k, q.device)
        if dv is None:
            dv = self._empty_like(v, q.device)
        if dgate is None:      # video tokens only (text tokens have no gate)
            dgate = self._empty_f32(q, q.shape[:-2] + (self.sizes.seq_len,))
        vsa2_attn_bwd(p, q, k, v, gate, self.map, o, lse, self.saved, d_o, dq, dk, dv, dgate, self.ws_bwd, stream=stream,
                      scratch=self._scratch("bwd_scratch_bytes", q.device, stream))
        return dq, dk, dv, dgate

    # A toy grid's calls wait for the host, and torch.empty takes 3.3 us: empty_like takes 1.5, new_empty
    # 2.4.  With the stream's plain handle (_current_stream) a training pass of 256 tokens takes 76 us instead of 93, of 2048 tokens 141 instead of 152.
    def _empty_f32(self, x, shape):
        torch = self.torch
        if type(x) is torch.Tensor:
            return x.new_empty(shape, dtype=torch.float32)
        return torch.empty(shape, dtype=torch.float32, device=x.device)

    def _empty_like(self, x, device):
        """An output tensor (contiguous, in the output type) of the shape of x.  (empty_like alone would keep the strides that x has in dimensions
        of size one.)"""
        torch = self.torch
        if type(x) is torch.Tensor and x.is_contiguous() and x.device == device:
            return torch.empty_like(x, dtype=self.out_torch_dtype, memory_format=torch.contiguous_format)
        return torch.empty(x.shape, dtype=self.out_torch_dtype, device=device)

    def _scratch(self, size, device, stream):
        """Scratch for one call of the bytes in attribute `size`, allocated on the stream the call runs on (its memory is then reused in
        that stream's order).  Where there is no room the call does without, and so do the next 16 calls, after a second refusal 32 and so
        on up to 1024 (a failing request makes the allocator empty its cache); meanwhile the attribute is 0."""
        torch, n, refused = self.torch, getattr(self, size), self._refused.get(size)
        if n == 0 and refused is not None:
            refused[2] -= 1
            if refused[2] < 0 and not torch.cuda.is_current_stream_capturing():
                n = refused[0]
        if n == 0:
            return None
        try:
            if stream is None:
                scratch = torch.empty(n, dtype=torch.uint8, device=device)
            else:
                if isinstance(stream, int):
                    stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
                with torch.cuda.stream(stream):
                    scratch = torch.empty(n, dtype=torch.uint8, device=device)
        except torch.cuda.OutOfMemoryError:
            calls = min(2 * refused[1], 1024) if refused is not None else 16
            self._refused[size] = [n, calls, calls]
            setattr(self, size, 0)
            return None
        if refused is not None:
            del self._refused[size]
            setattr(self, size, n)
        return scratch

    def check_status(self, stream=None):
        for name, ws in (("route", self.ws_route), ("fwd", self.ws_fwd), ("bwd", self.ws_bwd)):
            code = vsa2_device_status(ws, stream)
            if code != OK:
                raise Vsa2Error(code, f"device status after {name}")
