"""The residual stream between two products, as cases that can be timed: the operators `vsa2_residual_norm_fwd` / `vsa2_residual_norm_bwd`,
`vsa2_dropout`, `vsa2_int8_quantize` and `vsa2_int8_matmul`.

  norm_fwd  h = residual + dropout(x), y = h / sqrt(mean over the row of h^2 + eps) * weight; y leaves in bf16 or fp32, in e4m3 with a power-of-two
            scale for each 128 values of a row, or in int8 with a scale a row
  norm_bwd  gradients of y, and of h from the residual stream behind it -> of the residual, of x (through the dropout), and of the weight
  dropout   y = (residual +) x / (1 - p) where it is kept; the mask follows from a counter-based generator, nothing is stored
  quantize  a matrix -> int8 values with a scale a row
  matmul    C = A B^T of two such matrices, with a scale for each token and channel, and a bias

Where `own` is false every operator runs in its plain form, in fp32 torch operations; where it is true, through the library.
"""
import math

import torch

own = False

EPS = 1e-6


def _norm(name, op, rows, cols, *, f32=False, x_f32=False, out="bf16", residual=True, p=0.0):
    """f32: the residual stream (residual, h and their gradients) is fp32; x_f32: so is the branch x, and its gradient.  out (forward): what y leaves in;
    (backward): the type of y's gradient, bf16 or f32.  residual (backward): a gradient arrives at h from the stream."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "f32": f32, "x_f32": x_f32, "out": out, "residual": residual, "p": p}


def _dropout(name, rows, cols, p, *, f32=False, residual=False):
    return {"name": name, "op": "dropout", "rows": rows, "cols": cols, "p": p, "f32": f32, "residual": residual}


def _quantize(name, rows, cols, *, f32=False):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "f32": f32}


def _matmul(name, m, n, k, *, f32=False, bias=False):
    return {"name": name, "op": "matmul", "m": m, "n": n, "k": k, "f32": f32, "bias": bias}


def listed():
    return [
        # one token of a 40-head layer on its way to the int8 projection: a call's latency
        _norm("norm_one_token_int8", "norm_fwd", 1, 5120, out="int8"),
        # hidden states of 720p on their way to the fp8 projection
        _norm("norm_720p_fp8", "norm_fwd", 75600, 5120, out="fp8"),
        # training at 480p, a batch of two with text behind the videos: fp32 stream, dropout on the branch, y for the gate and for the projection
        _norm("norm_480p_train", "norm_fwd", 65972, 1536, f32=True, out="bf16+fp8", p=0.1),
        # training on the 2048-token clip
        _norm("norm_clip_bwd", "norm_bwd", 2048, 1536, p=0.1),
        # the gradients of the 480p step
        _norm("norm_480p_bwd", "norm_bwd", 65972, 1536, f32=True, p=0.1),
        # the clip's branch alone
        _dropout("dropout_clip", 2048, 1536, 0.1),
        # a branch of 720p added to its residual
        _dropout("dropout_720p_residual", 75600, 5120, 0.1, residual=True),
        # fp32 activations of odd sizes
        _quantize("int8_ragged_f32", 2025, 4600, f32=True),
        # the 40-head projection's weights
        _quantize("int8_weights", 15360, 5120),
        # one token against the 40-head projection: the weights' bytes are all
        _matmul("int8_one_token", 1, 15360, 5120, bias=True),
        # a clip of odd size, fp32 results
        _matmul("int8_ragged_f32_bias", 2025, 4603, 1530, f32=True, bias=True),
        # the 40-head projection of 720p
        _matmul("int8_720p", 75600, 15360, 5120),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one token to a 720p video, odd sizes."""
    cap = {"bytes": 0, "flops": 0}
    for c in listed():
        w = work(c)
        cap = {k: max(cap[k], w[k]) for k in cap}
    while True:
        op = rng.choice(["norm_fwd", "norm_fwd", "norm_bwd", "dropout", "quantize", "matmul", "matmul"])
        rows, cols = _log_int(rng, 1, 75600), 8 * _log_int(rng, 8, 1024) - rng.choice([0, 0, 0, 3])
        f32, p = rng.random() < 0.4, rng.choice([0.0, 0.1, rng.uniform(0.02, 0.6)])
        if op == "norm_fwd":
            c = _norm("", op, rows, cols, f32=f32, x_f32=f32 and rng.random() < 0.3, out=rng.choice(["bf16", "f32", "fp8", "int8", "int8", "bf16+fp8"]),
                      residual=rng.random() < 0.8, p=p)
        elif op == "norm_bwd":
            c = _norm("", op, rows, cols, f32=f32, x_f32=f32 and rng.random() < 0.3, out=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.8, p=p)
        elif op == "dropout":
            c = _dropout("", rows, cols, rng.uniform(0.02, 0.6), f32=f32, residual=rng.random() < 0.5)
        elif op == "quantize":
            c = _quantize("", rows, cols, f32=f32)
        else:
            c = _matmul("", _log_int(rng, 1, 40000), 8 * _log_int(rng, 8, 1920) - rng.choice([0, 0, 3]), _log_int(rng, 64, 8192), f32=rng.random() < 0.3,
                        bias=rng.random() < 0.5)
        del c["name"]
        w = work(c)
        if w["bytes"] <= 0.5 * cap["bytes"] and w["flops"] <= 0.5 * cap["flops"]:
            return c


def _outs(case):
    return case["out"].split("+")


def _branch_differs(case):
    """Whether the branch's gradient is not the residual's."""
    return _threshold(case["p"]) > 0 or case["f32"] != case["x_f32"]


def _room(rows, cols, dtype):
    """An 8-bit matrix whose rows begin on 16-byte boundaries."""
    return torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda").view(dtype)[:, :cols]


def _exponents(scales):
    """uint8 exponents + 127 as the powers of two that they stand for."""
    return scales.view(torch.float8_e8m0fnu)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = {"case": case}

    def randn(*shape, f32=False):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)

    def room(f32):
        return torch.empty(case["rows"], case["cols"], dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")

    if "p" in case:
        # seed and offset of the generator, kept on the device as a training program does that captures its step
        s["rng"] = torch.randint(0, 1 << 40, (2,), generator=gen, device="cuda")
    if op in ("norm_fwd", "norm_bwd"):
        rows, cols = case["rows"], case["cols"]
        channels = torch.exp(0.5 * randn(cols, f32=True))                                       # of unequal size
        s["w"] = 1.0 + 0.1 * randn(cols, f32=True)
    if op == "norm_fwd":
        s["x"] = randn(rows, cols, f32=case["x_f32"])
        s["r"] = randn(rows, cols, f32=case["f32"]).mul_(channels) if case["residual"] else None
        s["h"] = room(case["f32"] if case["residual"] else case["x_f32"])
        s["y"] = room("f32" in _outs(case)) if "bf16" in _outs(case) or "f32" in _outs(case) else None
        if "fp8" in _outs(case):
            s["fp8"] = _room(rows, cols, torch.float8_e4m3fn), torch.empty(-(-cols // 512), rows, 4, dtype=torch.uint8, device="cuda")
        if "int8" in _outs(case):
            s["int8"] = _room(rows, cols, torch.int8), torch.empty(rows, dtype=torch.float32, device="cuda")
    elif op == "norm_bwd":
        s["h"] = randn(rows, cols, f32=case["f32"]).mul_(channels)
        s["dy"] = randn(rows, cols, f32=case["out"] == "f32").mul_(1e-2)
        s["dh"] = randn(rows, cols, f32=case["f32"]).mul_(1e-2) if case["residual"] else None
        s["dr"], s["dx"] = room(case["f32"]), room(case["x_f32"]) if _branch_differs(case) else None
        s["dw"] = torch.empty(cols, dtype=torch.float32, device="cuda")
    elif op == "dropout":
        s["x"] = randn(case["rows"], case["cols"], f32=case["f32"])
        s["r"] = randn(case["rows"], case["cols"], f32=case["f32"]) if case["residual"] else None
        s["y"] = room(case["f32"])
    elif op == "quantize":
        s["x"] = randn(case["rows"], case["cols"], f32=case["f32"])
        s["x"] *= torch.exp(randn(case["rows"], 1, f32=True)).to(s["x"].dtype)
        s["int8"] = _room(case["rows"], case["cols"], torch.int8), torch.empty(case["rows"], dtype=torch.float32, device="cuda")
    else:
        m, n, k = case["m"], case["n"], case["k"]
        for name, rows in (("a", m), ("b", n)):
            values, scales = _room(rows, k, torch.int8), torch.empty(rows, dtype=torch.float32, device="cuda")
            for r in range(0, rows, 16384):
                values[r:r + 16384], scales[r:r + 16384] = _plain_int8(randn(min(16384, rows - r), k).float() * (k ** -0.5 if name == "b" else 1.0))
            s[name] = values, scales
        s["bias"] = 0.1 * randn(n, f32=True) if case["bias"] else None
        s["c"] = torch.empty(m, n, dtype=torch.float32 if case["f32"] else torch.bfloat16, device="cuda")
    return s


def _handles(s):
    """What a user's program makes once beside its inputs: workspaces."""
    from paper_2609_32882_b200 import binding as vb
    if "handles" not in s:
        c, h = s["case"], {}
        if c["op"] == "norm_bwd":
            h["workspace"] = torch.empty(vb.vsa2_residual_norm_bwd_workspace_bytes(c["rows"], c["cols"]), dtype=torch.uint8, device="cuda")
        if c["op"] == "matmul":
            h["workspace"] = vb.int8_matmul_workspace(c["m"], c["n"], c["k"], "cuda")
            h["a"], h["b"] = vb.Int8(*s["a"]), vb.Int8(*s["b"])
        if "fp8" in s:
            h["fp8"] = vb.Fp8(*s["fp8"])
        if "int8" in s:
            h["int8"] = vb.Int8(*s["int8"])
        s["handles"] = h
    return vb, s["handles"]


def _run_own(s):
    vb, handles = _handles(s)
    c = s["case"]
    op = c["op"]
    if op == "norm_fwd":
        vb.vsa2_residual_norm_fwd(s["x"], s["r"], s["w"], eps=EPS, h=s["h"], y=s["y"], y_fp8=handles.get("fp8"), y_int8=handles.get("int8"), p=c["p"],
                                  rng=s["rng"])
        return _forward_outputs(s["h"], s["y"], s.get("fp8"), s.get("int8"))
    if op == "norm_bwd":
        vb.vsa2_residual_norm_bwd(s["h"], s["dy"], s["dh"], s["w"], eps=EPS, d_residual=s["dr"], dx=s["dx"], d_weight=s["dw"], workspace=handles["workspace"],
                                  p=c["p"], rng=s["rng"])
        return {"dr": s["dr"], "dx": s["dx"], "dw": s["dw"]}      # (dx None: the residual's is the branch's too)
    if op == "dropout":
        vb.vsa2_dropout(s["x"], s["y"], c["p"], s["rng"], residual=s["r"])
        return {"y": s["y"]}
    if op == "quantize":
        vb.vsa2_int8_quantize(s["x"], handles["int8"])
        return {"values": s["int8"][0], "scales": s["int8"][1]}
    vb.vsa2_int8_matmul(handles["a"], handles["b"], s["c"], handles["workspace"], bias=s["bias"])
    return {"c": s["c"]}


def _forward_outputs(h, y, fp8, int8):
    out = {"h": h}
    if y is not None:
        out["y"] = y
    if fp8 is not None:
        out["fp8"], out["fp8_scales"] = fp8[0], _exponents(fp8[1])
    if int8 is not None:
        out["int8"], out["int8_scales"] = int8
    return out


def _threshold(p):
    """The mask keeps an element whose 16 bits are at least this."""
    return min(65535, int(p * 65536 + 0.5))


def _kept(rng, rows, cols, p):
    """Which elements a dropout keeps: 16 bits each of the Philox generator (4 x 32 bits, 10 rounds; Salmon et al., 2011), whose key is the seed and whose
    counter is (column / 8, row, offset); truth values [rows, cols]."""
    low = 0xffffffff
    octs = -(-cols // 8)
    a = torch.arange(octs, device="cuda").expand(rows, octs)
    b = torch.arange(rows, device="cuda").unsqueeze(1).expand(rows, octs)
    c, d = rng[1] & low, (rng[1] >> 32) & low
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        u, v = a * 0xD2511F53, c * 0xCD9E8D57                          # 64 bits, beyond which nothing is wanted
        a, b, c, d = ((v >> 32) & low) ^ b ^ k0, v & low, ((u >> 32) & low) ^ d ^ k1, u & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([a, b, c, d], dim=-1)
    pieces = torch.stack([words & 0xffff, words >> 16], dim=-1)        # of eight neighbours, in their order
    return (pieces >= _threshold(p)).view(rows, octs * 8)[:, :cols]


def _dropped(x, rng, p):
    if _threshold(p) == 0:
        return x
    return torch.where(_kept(rng, *x.shape, p), x * (65536.0 / (65536 - _threshold(p))), 0.0)


def _plain_fp8(x):
    """Values (e4m3) of an fp32 matrix and their scales (exponent + 127, uint8 [ceil(cols / 512), rows, 4])."""
    rows, cols = x.shape
    kb = -(-cols // 128)
    a = torch.nn.functional.pad(x.abs(), (0, kb * 128 - cols)).view(rows, kb, 128).amax(dim=-1)
    mantissa, e = torch.frexp(a)                                       # a = mantissa 2^e, 448 = 0.875 2^9
    e = torch.where(a > 0, torch.where(mantissa > 0.875, e - 8, e - 9), -127).clamp(-127, 127)
    values = torch.ldexp(x, -e.repeat_interleave(128, dim=1)[:, :cols]).to(torch.float8_e4m3fn)
    return values, torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -kb % 4)).view(rows, -1, 4).transpose(0, 1).contiguous()


def _plain_int8(x):
    """Values of an fp32 matrix and its rows' scales."""
    top = x.abs().amax(dim=1).clamp(min=2.0 ** -100)
    # (a division: torch takes a number over a tensor as the reciprocal times the number, which is rounded twice)
    return torch.round(x * torch.div(torch.full_like(top, 127.0), top).unsqueeze(1)).to(torch.int8), top / 127.0


def run(state):
    if own:
        return _run_own(state)
    s, c = state, state["case"]
    op = c["op"]
    if op == "norm_fwd":
        h = _dropped(s["x"].float(), s["rng"], c["p"])
        if s["r"] is not None:
            h = s["r"].float() + h
        stored = h.to(s["h"].dtype)
        h = stored.float()                                             # the norm is that of what is stored
        factor = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
        v = h * s["w"]
        fp8 = int8 = None
        if "fp8" in s:
            fp8 = _plain_fp8(v * factor)
        if "int8" in s:
            int8 = _plain_int8(v)                                      # the row's factor goes into its scale
            int8 = int8[0], int8[1] * factor.squeeze(1)
        return _forward_outputs(stored, None if s["y"] is None else (v * factor).to(s["y"].dtype), fp8, int8)
    if op == "norm_bwd":
        h, dy = s["h"].float(), s["dy"].float()
        factor = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
        hat, g = h * factor, dy * s["w"]
        d = factor * (g - hat * (g * hat).mean(dim=1, keepdim=True))
        if s["dh"] is not None:
            d = d + s["dh"].float()
        dx = _dropped(d, s["rng"], c["p"]).to(s["dx"].dtype) if s["dx"] is not None else None
        return {"dr": d.to(s["dr"].dtype), "dx": dx, "dw": (dy * hat).sum(dim=0)}
    if op == "dropout":
        y = _dropped(s["x"].float(), s["rng"], c["p"])
        return {"y": (y if s["r"] is None else s["r"].float() + y).to(s["y"].dtype)}
    if op == "quantize":
        values, scales = _plain_int8(s["x"].float())
        return {"values": values, "scales": scales}
    y = (s["a"][0].float() @ s["b"][0].float().T) * s["a"][1].unsqueeze(1) * s["b"][1]
    return {"c": (y if s["bias"] is None else y + s["bias"]).to(s["c"].dtype)}


def work(case):
    op = case["op"]
    if op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * (k + 4) + m * n * (4 if case["f32"] else 2) + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    rows, elems, size = case["rows"], case["rows"] * case["cols"], 4 if case["f32"] else 2
    if op == "quantize":
        return {"bytes": elems * (size + 1) + 4 * rows, "flops": 2 * elems}
    if op == "dropout":
        return {"bytes": elems * size * (3 if case["residual"] else 2), "flops": 8 * elems}
    x_size, drop = 4 if case["x_f32"] else 2, 7 if _threshold(case["p"]) else 0
    if op == "norm_fwd":
        outs = {"bf16": 2 * elems, "f32": 4 * elems, "fp8": elems * (1 + 1 / 128), "int8": elems + 4 * rows}
        stream = 2 * size * elems if case["residual"] else x_size * elems
        return {"bytes": x_size * elems + stream + sum(outs[o] for o in _outs(case)) + 4 * case["cols"], "flops": (6 + drop) * elems}
    grads = elems * (4 if case["out"] == "f32" else 2) + size * elems * (3 if case["residual"] else 2) + (x_size * elems if _branch_differs(case) else 0)
    return {"bytes": grads + 8 * case["cols"], "flops": (12 + drop) * elems}


def _exact_factors(rng, rows, cols, p):
    """What a dropout multiplies by, fp64 [rows, cols]: the generator's products by halves of 16 bits."""
    t = _threshold(p)
    if t == 0:
        return torch.ones(1, 1, dtype=torch.float64, device="cuda")
    octs = (cols + 7) // 8
    seed, offset = (int(v) for v in rng.tolist())

    def times(x, m):                    # high and low word of a product of two words
        x0, x1, m0, m1 = x % 65536, x // 65536, m % 65536, m // 65536
        middle = x1 * m0 + (x0 * m0) // 65536
        other = x0 * m1 + middle % 65536
        return x1 * m1 + middle // 65536 + other // 65536, (other % 65536) * 65536 + (x0 * m0) % 65536

    grid = torch.zeros(rows, octs, dtype=torch.int64, device="cuda")
    state = [grid + torch.arange(octs, device="cuda"), grid + torch.arange(rows, device="cuda")[:, None], grid + offset % 2 ** 32, grid + offset // 2 ** 32]
    for i in range(10):
        keys = (seed + i * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32
        (hi0, lo0), (hi1, lo1) = times(state[0], 0xD2511F53), times(state[2], 0xCD9E8D57)
        state = [hi1.bitwise_xor(state[1]).bitwise_xor(keys[0]), lo1, hi0.bitwise_xor(state[3]).bitwise_xor(keys[1]), lo0]
    factors = torch.empty(rows, octs * 8, dtype=torch.float64, device="cuda")
    for j in range(8):
        bits = state[j // 2] // 65536 if j % 2 else state[j // 2] % 65536
        factors[:, j::8] = torch.where(bits < t, 0.0, 65536.0 / (65536 - t))
    return factors[:, :cols]


def exact(case, seed):
    """The same outputs from the definitions in 64 bits, in pieces of rows."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "matmul":
        b = s["b"][0].double() * s["b"][1].double().unsqueeze(1)
        c = torch.empty(case["m"], case["n"], dtype=torch.float64, device="cuda")
        for r in range(0, case["m"], 16384):
            c[r:r + 16384] = (s["a"][0][r:r + 16384].double() * s["a"][1][r:r + 16384].double().unsqueeze(1)) @ b.T
        return {"c": c if s["bias"] is None else c + s["bias"].double()}
    if op == "quantize":
        return {"values": None, "scales": s["x"].double().abs().max(dim=1).values / 127}
    rows, cols = case["rows"], case["cols"]
    factors = _exact_factors(s["rng"], rows, cols, case["p"])
    if op == "dropout":
        y = s["x"].double() * factors
        return {"y": y if s["r"] is None else y + s["r"]}
    w = s["w"].double()
    if op == "norm_fwd":
        h = s["x"].double() * factors
        if s["r"] is not None:
            h += s["r"]
        stored = h.to(s["h"].dtype).double()
        length = torch.linalg.vector_norm(stored, dim=1, keepdim=True)
        y = stored * w / torch.sqrt(length * length / cols + EPS)
        fp8 = int8 = None
        if "fp8" in s:
            parts = [y[:, i:i + 128] for i in range(0, cols, 128)]
            # (a maximum of 448 times a power of two is common, one a hair above it is 1.7e-7 away: the logarithm's own error is neither)
            e = [torch.ceil(torch.log2(b.abs().amax(dim=1, keepdim=True) / 448.0) - 1e-12).clamp(min=-127.0) for b in parts]
            scales = torch.full((rows, -(-cols // 512) * 4), 2.0 ** -127, dtype=torch.float64, device="cuda")      # (behind the last block: exponent byte 0)
            scales[:, :len(e)] = torch.exp2(torch.cat(e, dim=1))
            fp8 = torch.cat([b / torch.exp2(v) for b, v in zip(parts, e)], dim=1), scales.view(rows, -1, 4).transpose(0, 1).contiguous()
        if "int8" in s:
            int8 = None, y.abs().max(dim=1).values / 127
        out = {"h": h}
        if s["y"] is not None:
            out["y"] = y
        if fp8 is not None:
            out["fp8"], out["fp8_scales"] = fp8
        if int8 is not None:
            out["int8"], out["int8_scales"] = int8
        return out
    h, dy = s["h"].double(), s["dy"].double()
    ms = h.square().sum(dim=1, keepdim=True) / cols + EPS
    dw = (dy * h / ms.sqrt()).sum(dim=0)
    g = dy * w
    d = g / ms.sqrt() - h * (g * h).sum(dim=1, keepdim=True) / (cols * ms * ms.sqrt())
    if s["dh"] is not None:
        d += s["dh"]
    return {"dr": d, "dx": d * factors if s["dx"] is not None else None, "dw": dw}
