"""The work between a layer's hidden states and its attention, as cases that can be timed: the operators `vsa2_rope_apply`,
`vsa2_qkv_fwd` / `vsa2_qkv_bwd`, `vsa2_fp8_quantize` and `vsa2_fp8_matmul`.

  rope      rotary positions on (time, height, width): y = R(position) x, or with the inverse rotation (the gradient)
  qkv_fwd   rows of a packed projection [batch, tokens, (Hq + 2 Hkv) D] -> q, k (norm of each head, weight, rotation) and v as
            [batch, heads, tokens, D]
  qkv_bwd   gradients of q, k, v -> gradient of the packed rows and of the two norm weights
  quantize  a matrix -> e4m3 values with a power-of-two scale for each block of 128 (of a row, or of 128 rows), and its transpose likewise
  matmul    C = A B^T of two such matrices

Where `own` is false every operator runs in its plain form, in fp32 torch operations; where it is true, through the library.
"""
import math

import torch

own = False

PAIRS, HALVES = "pairs", "halves"


def _rope(name, batch, heads, grid, dim, channels, *, layout=PAIRS, inverse=False, f32=False, text=0, listed_positions=False,
          token_major=False):
    """channels: how many channels turn with t, h and w; text: rows behind the grid that do not turn; listed_positions: every
    token's position is read from a list (pictures of several sizes in one row) instead of following from the grid; token_major: x is
    [batch, tokens, heads, dim] in memory."""
    return {"name": name, "op": "rope", "batch": batch, "heads": heads, "t": grid[0], "h": grid[1], "w": grid[2], "dim": dim,
            "ct": channels[0], "ch": channels[1], "cw": channels[2], "layout": layout, "inverse": inverse, "f32": f32, "text": text,
            "positions": listed_positions, "token_major": token_major}


def _qkv(name, op, batch, heads_q, heads_kv, grid, dim, channels, *, layout=PAIRS, text=0, f32=False):
    """f32 (backward): the gradients come, and leave, in fp32."""
    return {"name": name, "op": op, "batch": batch, "heads_q": heads_q, "heads_kv": heads_kv, "t": grid[0], "h": grid[1], "w": grid[2],
            "dim": dim, "ct": channels[0], "ch": channels[1], "cw": channels[2], "layout": layout, "text": text, "f32": f32}


def _quantize(name, rows, cols, *, form="rows", squares=False, f32=False):
    """form: "rows", "both" (the transpose too); squares: blocks of 128 x 128 instead of 1 x 128."""
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "form": form, "squares": squares, "f32": f32}


def _matmul(name, m, n, k, *, f32=False, squares=True):
    """squares: B has one scale for 128 x 128 values (weights), else one for 1 x 128 like A."""
    return {"name": name, "op": "matmul", "m": m, "n": n, "k": k, "f32": f32, "squares": squares}


def listed():
    return [
        # the toy grid of the tests: a call's latency
        _rope("rope_toy", 1, 2, (4, 8, 8), 64, (16, 24, 24)),
        # the queries of a 720p layer, projected without a norm
        _rope("rope_720p", 1, 40, (21, 45, 80), 128, (44, 42, 42)),
        # gradients of keys over pictures of several sizes, positions from a list, halves of a head as pairs, token-major input
        _rope("rope_pictures_grad_f32", 2, 16, (13, 27, 47), 64, (0, 32, 32), layout=HALVES, inverse=True, f32=True,
              listed_positions=True, token_major=True),
        # the toy grid again
        _qkv("qkv_toy_fwd", "qkv_fwd", 1, 2, 2, (4, 8, 8), 64, (16, 24, 24)),
        # a whole 40-head layer of 720p video: the repository's benchmark shape
        _qkv("qkv_720p_fwd", "qkv_fwd", 1, 40, 40, (21, 45, 80), 128, (44, 42, 42)),
        # training on the 2048-token clip
        _qkv("qkv_clip_bwd", "qkv_bwd", 1, 12, 12, (8, 16, 16), 128, (16, 56, 56)),
        # 480p training with grouped heads, text behind the video, a batch of two
        _qkv("qkv_480p_text_bwd", "qkv_bwd", 2, 12, 3, (21, 30, 52), 128, (44, 42, 42), text=226),
        # hidden states of 720p before the projection
        _quantize("fp8_hidden_720p", 75600, 5120),
        # gradients of the clip's packed rows for both of their products, odd sizes
        _quantize("fp8_gradient_both", 2025, 4600, form="both"),
        # one row (a time step's embedding, one token) against the 40-head projection: the weights' bytes are all
        _matmul("fp8_one_row", 1, 15360, 5120),
        # the 40-head projection of 720p
        _matmul("fp8_720p", 75600, 15360, 5120),
        # gradient of the 480p projection's weights: a long sum, fp32
        _matmul("fp8_weight_gradient_480p", 2304, 1536, 32760, f32=True, squares=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: toy grids to 720p, one row to a whole video, odd sizes."""
    cap = {"bytes": 0, "flops": 0}
    for c in listed():
        w = work(c)
        cap = {k: max(cap[k], w[k]) for k in cap}
    while True:
        op = rng.choice(["rope", "qkv_fwd", "qkv_bwd", "quantize", "matmul"])
        grid = (_log_int(rng, 1, 33), _log_int(rng, 4, 45), _log_int(rng, 4, 80))
        dim = rng.choice([64, 128, 128])
        channels = rng.choice([(16, 24, 24), (0, 32, 32), (20, 22, 22)] if dim == 64 else [(44, 42, 42), (16, 56, 56), (32, 32, 32)])
        layout = rng.choice([PAIRS, HALVES])
        if layout == HALVES and sum(channels) % 16:
            continue
        batch, text = rng.choice([1, 1, 2, 3]), rng.choice([0, 0, rng.randint(1, 300)])
        if op == "rope":
            c = _rope("", batch, _log_int(rng, 1, 40), grid, dim, channels, layout=layout, inverse=rng.random() < 0.5,
                      f32=rng.random() < 0.4, text=text, listed_positions=rng.random() < 0.3, token_major=rng.random() < 0.4)
        elif op in ("qkv_fwd", "qkv_bwd"):
            kv = _log_int(rng, 1, 40)
            hq = kv * rng.choice([1, 1, 2, 4])
            c = _qkv("", op, batch, hq, kv, grid, dim, channels, layout=layout, text=text,
                     f32=op == "qkv_bwd" and rng.random() < 0.4)
            if hq > 40:
                continue
        elif op == "quantize":
            c = _quantize("", _log_int(rng, 1, 75600), _log_int(rng, 64, 15360), form=rng.choice(["rows", "both"]),
                          squares=rng.random() < 0.4, f32=rng.random() < 0.3)
        else:
            c = _matmul("", _log_int(rng, 1, 40000), 8 * _log_int(rng, 8, 1920) - rng.choice([0, 0, 3]), _log_int(rng, 64, 8192),
                        f32=rng.random() < 0.3, squares=rng.random() < 0.6)
        del c["name"]
        w = work(c)
        if w["bytes"] <= 0.5 * cap["bytes"] and w["flops"] <= 0.5 * cap["flops"]:
            return c


def _tokens(case):
    return case["t"] * case["h"] * case["w"] + case["text"]


def _grid_positions(case):
    """(t, h, w) of the grid's tokens in raster order; int64 [T H W, 3]."""
    t, h, w = case["t"], case["h"], case["w"]
    i = torch.arange(t * h * w, device="cuda")
    return torch.stack([i // (h * w), i // w % h, i % w], dim=-1)


def _plain_quantize(x, squares):
    """Values (e4m3, of x's shape) and exponents + 127 (uint8, [rows, blocks of 128 columns]) of an fp32 matrix."""
    rows, cols = x.shape
    kb = -(-cols // 128)
    fine = torch.isfinite(x)
    a = torch.nn.functional.pad(torch.where(fine, x, 0.0).abs(), (0, kb * 128 - cols)).view(rows, kb, 128).amax(dim=-1)
    if squares:
        rb = -(-rows // 128)
        a = torch.nn.functional.pad(a, (0, 0, 0, rb * 128 - rows)).view(rb, 128, kb).amax(dim=1)
        a = a.repeat_interleave(128, dim=0)[:rows]
    mantissa, e = torch.frexp(a)                               # a = mantissa 2^e, 448 = 0.875 2^9
    e = torch.where(mantissa > 0.875, e - 8, e - 9)
    e = torch.where(a > 0, e, -127).clamp(-127, 127)
    scaled = torch.ldexp(x, -e.repeat_interleave(128, dim=1)[:, :cols])
    return torch.where(fine, scaled, float("nan")).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _pack_scales(e):
    """[rows, blocks] -> [ceil(blocks / 4), rows, 4], the library's order; what is beyond the last block is zero."""
    rows, kb = e.shape
    return torch.nn.functional.pad(e, (0, -kb % 4)).view(rows, -1, 4).transpose(0, 1).contiguous()


def _unpack_scales(s, cols):
    """The scale of every value of a row, fp32 [rows, cols]."""
    e = s.transpose(0, 1).reshape(s.shape[1], -1).to(torch.int32) - 127
    return torch.ldexp(torch.ones((), device=s.device), e).repeat_interleave(128, dim=1)[:, :cols]


def _room(rows, cols):
    """An e4m3 matrix whose rows begin on 16-byte boundaries."""
    return torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = {"case": case}

    def randn(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    if op in ("rope", "qkv_fwd", "qkv_bwd"):
        b, n, d = case["batch"], _tokens(case), case["dim"]
        # frequencies of the pairs, axis by axis, and the axis of each
        s["freq"] = torch.tensor([1e4 ** (-2.0 * j / c) for c in (case["ct"], case["ch"], case["cw"]) for j in range(c // 2)], device="cuda")
        s["axis"] = torch.tensor([a for a, c in enumerate((case["ct"], case["ch"], case["cw"])) for j in range(c // 2)], device="cuda")
        s["positions"] = None
        s["grid"] = _grid_positions(case)
    if op == "rope":
        dtype, heads = torch.float32 if case["f32"] else torch.bfloat16, case["heads"]
        if case["token_major"]:
            s["x"] = randn(b, n, heads, d, dtype=dtype).transpose(1, 2)
        else:
            s["x"] = randn(b, heads, n, d, dtype=dtype)
        if case["positions"]:
            # pictures of 32 x 20 patches, one behind the other, each with its own index on the first axis; another start per batch entry
            i = torch.arange(n, device="cuda") + torch.randint(0, 640, (b, 1), generator=gen, device="cuda")
            s["positions"] = torch.stack([i // 640, i // 20 % 32, i % 20], dim=-1).to(torch.int32)
        s["y"] = torch.empty(b, heads, n, d, dtype=dtype, device="cuda")
    elif op in ("qkv_fwd", "qkv_bwd"):
        hq, hk = case["heads_q"], case["heads_kv"]
        s["x"] = randn(b, n, (hq + 2 * hk) * d)
        s["x"] *= torch.exp(0.5 * randn((hq + 2 * hk) * d, dtype=torch.float32)).bfloat16()      # channels of unequal size
        s["w"] = [1.0 + 0.1 * randn(d, dtype=torch.float32) for _ in range(2)]
        if op == "qkv_fwd":
            s["y"] = [torch.empty(b, h, n, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hk)]
        else:
            dtype = torch.float32 if case["f32"] else torch.bfloat16
            s["dy"] = [randn(b, h, n, d, dtype=dtype) * 1e-2 for h in (hq, hk, hk)]
            s["dx"] = torch.empty(b, n, (hq + 2 * hk) * d, dtype=dtype, device="cuda")
            s["dw"] = [torch.empty(d, dtype=torch.float32, device="cuda") for _ in range(2)]
    elif op == "quantize":
        rows, cols = case["rows"], case["cols"]
        s["x"] = randn(rows, cols, dtype=torch.float32 if case["f32"] else torch.bfloat16)
        s["x"] *= torch.exp(randn(rows, 1, dtype=torch.float32)).to(s["x"].dtype)
        shapes = [(rows, cols)] + ([(cols, rows)] if case["form"] == "both" else [])
        s["values"] = [_room(*sh) for sh in shapes]
        s["scales"] = [torch.empty(-(-sh[1] // 512), sh[0], 4, dtype=torch.uint8, device="cuda") for sh in shapes]
    else:
        m, n, k = case["m"], case["n"], case["k"]
        for name, rows, squares, size in (("a", m, False, 1.0), ("b", n, case["squares"], k ** -0.5)):
            x = randn(rows, k) * size
            s[name] = _room(rows, k)
            for r in range(0, rows, 16384):
                v, e = _plain_quantize(x[r:r + 16384].float(), squares)
                s[name].view(torch.uint8)[r:r + 16384] = v.view(torch.uint8)
                s.setdefault(name + "_e", []).append(e)
            s[name + "_scales"] = _pack_scales(torch.cat(s.pop(name + "_e")))
        s["c"] = torch.empty(m, n, dtype=torch.float32 if case["f32"] else torch.bfloat16, device="cuda")
    return s


def _handles(s):
    """What a user's program makes once beside its inputs: plan and workspace."""
    from paper_2609_32882_b200 import binding as vb
    if "handles" not in s:
        c, h = s["case"], {}
        if "freq" in s:
            h["rope"] = vb.vsa2_rope_plan(c["dim"], (c["ct"], c["ch"], c["cw"]),
                                          layout=vb.ROPE_HALVES if c["layout"] == HALVES else vb.ROPE_PAIRS)
        if c["op"] == "qkv_bwd":
            h["workspace"] = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(c["dim"]), dtype=torch.uint8, device="cuda")
        if c["op"] == "matmul":
            h["workspace"] = vb.fp8_matmul_workspace(c["m"], c["n"], c["k"], "cuda")
        s["handles"] = h
    return vb, s["handles"]


def _packed_heads(x, case):
    """Views [batch, heads, tokens, D] of the packed rows."""
    d, hq, hk = case["dim"], case["heads_q"], case["heads_kv"]
    h = x.unflatten(-1, (hq + 2 * hk, d)).transpose(1, 2)
    return [h[:, :hq], h[:, hq:hq + hk], h[:, hq + hk:]]


def _run_own(s):
    vb, h = _handles(s)
    c = s["case"]
    op = c["op"]
    grid = (c["t"], c["h"], c["w"]) if "t" in c else None
    if op == "rope":
        vb.vsa2_rope_apply(h["rope"], s["x"], s["y"], grid=grid, positions=s["positions"], inverse=c["inverse"])
        return {"y": s["y"]}
    if op == "qkv_fwd":
        vb.vsa2_qkv_fwd(h["rope"], _packed_heads(s["x"], c), s["y"], *s["w"], grid=grid)
        return dict(zip(("q", "k", "v"), s["y"]))
    if op == "qkv_bwd":
        vb.vsa2_qkv_bwd(h["rope"], _packed_heads(s["x"], c), s["dy"], _packed_heads(s["dx"], c), *s["w"], *s["dw"], h["workspace"], grid=grid)
        return {"dx": s["dx"], "dwq": s["dw"][0], "dwk": s["dw"][1]}
    if op == "quantize":
        forms = [vb.Fp8(v, e) for v, e in zip(s["values"], s["scales"])]
        vb.vsa2_fp8_quantize(s["x"], forms[0], forms[1] if len(forms) > 1 else None, squares=c["squares"])
        return {"values": s["values"], "scales": s["scales"]}
    vb.vsa2_fp8_matmul(vb.Fp8(s["a"], s["a_scales"]), vb.Fp8(s["b"], s["b_scales"]), s["c"], h["workspace"])
    return {"c": s["c"]}


def _cos_sin(s):
    """cos and sin of every pair's angle, fp32 [batch or nothing, 1, tokens, pairs]; rows behind the grid do not turn."""
    c = s["case"]
    at = s["positions"] if s["positions"] is not None else torch.nn.functional.pad(s["grid"], (0, 0, 0, c["text"]))
    angle = at.float()[..., s["axis"]] * s["freq"]
    return torch.cos(angle).unsqueeze(-3), torch.sin(angle).unsqueeze(-3)


def _turn(x, cos, sin, layout):
    """x [.., tokens, D] fp32 turned by the angles."""
    p = cos.shape[-1]
    if layout == HALVES:
        a, b = x[..., :p], x[..., p:2 * p]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., 2 * p:]], dim=-1)
    a, b = x[..., 0:2 * p:2], x[..., 1:2 * p:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), x[..., 2 * p:]], dim=-1)


def _normed(x):
    """Every head's row over its root mean square, and the factor."""
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6)
    return x * r, r


def _norm_grad(x, w, dy, cos, sin, layout):
    g = _turn(dy.float(), cos, -sin, layout)
    hat, r = _normed(x.float())
    wg = g * w
    return r * (wg - hat * (wg * hat).mean(dim=-1, keepdim=True)), (g * hat).sum(dim=(0, 1, 2))


def run(state):
    if own:
        return _run_own(state)
    s, c = state, state["case"]
    op = c["op"]
    if op == "rope":
        cos, sin = _cos_sin(s)
        return {"y": _turn(s["x"].float(), cos, -sin if c["inverse"] else sin, c["layout"]).to(s["y"].dtype)}
    if op == "qkv_fwd":
        cos, sin = _cos_sin(s)
        xq, xk, xv = _packed_heads(s["x"], c)
        return {"q": _turn(_normed(xq.float())[0] * s["w"][0], cos, sin, c["layout"]).bfloat16(),
                "k": _turn(_normed(xk.float())[0] * s["w"][1], cos, sin, c["layout"]).bfloat16(), "v": xv.contiguous()}
    if op == "qkv_bwd":
        cos, sin = _cos_sin(s)
        xq, xk, _ = _packed_heads(s["x"], c)
        dxq, dwq = _norm_grad(xq, s["w"][0], s["dy"][0], cos, sin, c["layout"])
        dxk, dwk = _norm_grad(xk, s["w"][1], s["dy"][1], cos, sin, c["layout"])
        dx = torch.cat([dxq, dxk, s["dy"][2].float()], dim=1).transpose(1, 2).flatten(2)
        return {"dx": dx.to(s["dx"].dtype), "dwq": dwq, "dwk": dwk}
    if op == "quantize":
        x = s["x"].float()
        values, e = _plain_quantize(x, c["squares"])
        if c["form"] == "rows":
            return {"values": [values], "scales": [_pack_scales(e)]}
        values_t, e_t = _plain_quantize(x.T, c["squares"])
        return {"values": [values, values_t], "scales": [_pack_scales(e), _pack_scales(e_t)]}
    a = s["a"].float() * _unpack_scales(s["a_scales"], c["k"])
    b = s["b"].float() * _unpack_scales(s["b_scales"], c["k"])
    return {"c": (a @ b.T).to(s["c"].dtype)}


def work(case):
    op = case["op"]
    if op == "rope":
        elems = case["batch"] * case["heads"] * _tokens(case) * case["dim"]
        nbytes = 2 * elems * (4 if case["f32"] else 2)
        if case["positions"]:
            nbytes += 12 * case["batch"] * _tokens(case)
        return {"bytes": nbytes, "flops": 3 * elems}
    if op in ("qkv_fwd", "qkv_bwd"):
        rows = case["batch"] * _tokens(case) * case["dim"]
        q, kv = rows * case["heads_q"], rows * case["heads_kv"]
        if op == "qkv_fwd":
            return {"bytes": 4 * (q + 2 * kv) + 8 * case["dim"], "flops": 7 * (q + kv)}
        grad = 4 if case["f32"] else 2
        return {"bytes": 2 * (q + kv) + 2 * grad * (q + 2 * kv) + 16 * case["dim"], "flops": 14 * (q + kv)}
    if op == "quantize":
        elems, forms = case["rows"] * case["cols"], 2 if case["form"] == "both" else 1
        return {"bytes": elems * ((4 if case["f32"] else 2) + forms + forms / 128), "flops": 2 * elems * forms}
    m, n, k = case["m"], case["n"], case["k"]
    return {"bytes": (m + n) * k * (1 + 1 / 128) + m * n * (4 if case["f32"] else 2), "flops": 2 * m * n * k}


def exact(case, seed):
    """The same outputs from the definitions in 64 bits: rotations as products of complex numbers, gradients of the norm through its
    Jacobian, scales from logarithms.  Head by head, as 64-bit copies of everything would not fit."""
    s = prepare(case, seed)
    op = case["op"]
    if op in ("rope", "qkv_fwd", "qkv_bwd"):
        n, axes = _tokens(case), (case["ct"], case["ch"], case["cw"])
        pairs = sum(axes) // 2
        if s["positions"] is not None:
            place = s["positions"].double()
        else:
            place = torch.zeros(1, n, 3, dtype=torch.float64, device="cuda")
            place[0, :n - case["text"]] = s["grid"].double()
        parts = []
        for a, c in enumerate(axes):
            exponent = -torch.arange(0, c, 2, dtype=torch.float64, device="cuda") / max(c, 1)
            parts.append(place[:, :, a:a + 1] * torch.pow(torch.tensor(1e4, dtype=torch.float64, device="cuda"), exponent))
        angle = torch.cat(parts, dim=-1)
        if case["layout"] == HALVES:
            first, second = torch.arange(pairs, device="cuda"), torch.arange(pairs, 2 * pairs, device="cuda")
        else:
            first, second = torch.arange(0, 2 * pairs, 2, device="cuda"), torch.arange(1, 2 * pairs, 2, device="cuda")

        def rotate(x, sign):              # x [batch, tokens, D] in 64 bits
            z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), sign * angle)
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y

    if op == "rope":
        y = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
        for h in range(case["heads"]):
            y[:, h] = rotate(s["x"][:, h].double(), -1.0 if case["inverse"] else 1.0)
        return {"y": y}
    if op in ("qkv_fwd", "qkv_bwd"):
        hq, hk, d = case["heads_q"], case["heads_kv"], case["dim"]
        x = s["x"].view(case["batch"], n, hq + 2 * hk, d)
    if op == "qkv_fwd":
        out = [torch.empty(case["batch"], h, n, d, dtype=torch.float64, device="cuda") for h in (hq, hk, hk)]
        for h in range(hq + 2 * hk):
            xh = x[:, :, h].double()
            if h >= hq + hk:
                out[2][:, h - hq - hk] = xh
                continue
            w = s["w"][0 if h < hq else 1].double()
            xh = xh / torch.sqrt(xh.square().sum(dim=-1, keepdim=True) / d + 1e-6) * w
            out[0 if h < hq else 1][:, h if h < hq else h - hq] = rotate(xh, 1.0)
        return {"q": out[0], "k": out[1], "v": out[2]}
    if op == "qkv_bwd":
        dx = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        dw = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2)]
        for h in range(hq + 2 * hk):
            if h >= hq + hk:
                dx[:, :, h] = s["dy"][2][:, h - hq - hk].double()
                continue
            part, i = (0, h) if h < hq else (1, h - hq)
            xh, g = x[:, :, h].double(), rotate(s["dy"][part][:, i].double(), -1.0)
            ms = xh.square().sum(dim=-1, keepdim=True) / d + 1e-6
            dw[part] += (g * xh / ms.sqrt()).sum(dim=(0, 1))
            g = g * s["w"][part].double()
            dx[:, :, h] = g / ms.sqrt() - xh * (g * xh).sum(dim=-1, keepdim=True) / (d * ms * ms.sqrt())
        return {"dx": dx.flatten(2), "dwq": dw[0], "dwk": dw[1]}
    if op == "quantize":
        values = []
        for transposed in ([False, True] if case["form"] == "both" else [False]):
            x = s["x"].T if transposed else s["x"]
            v = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            step = 128 if case["squares"] else 1
            for c0 in range(0, x.shape[1], 128):
                block = x[:, c0:c0 + 128].double()
                top = block.abs().amax(dim=1)
                if step > 1:
                    groups = torch.arange(x.shape[0], device="cuda") // step
                    top = torch.zeros(int(groups[-1]) + 1, dtype=torch.float64, device="cuda").scatter_reduce(0, groups, top, "amax")[groups]
                # (a maximum of 448 times a power of two is common, one a hair above it is 1.7e-7 away: the logarithm's own error is neither)
                v[:, c0:c0 + 128] = block / torch.exp2(torch.ceil(torch.log2(top / 448.0) - 1e-12).clamp(min=-127.0)).unsqueeze(1)
            values.append(v)
        return {"values": values, "scales": [None] * len(values)}

    def wide(v, e):
        x = v.double()
        for i in range(0, v.shape[1], 128):
            x[:, i:i + 128] *= torch.exp2(e[i // 512, :, i // 128 % 4].double() - 127.0).unsqueeze(1)
        return x

    b = wide(s["b"], s["b_scales"])
    c = torch.empty(case["m"], case["n"], dtype=torch.float64, device="cuda")
    for r in range(0, case["m"], 16384):
        c[r:r + 16384] = wide(s["a"][r:r + 16384], s["a_scales"][:, r:r + 16384]) @ b.T
    return {"c": c}
