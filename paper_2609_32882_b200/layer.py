"""One self-attention layer from its hidden states on: the library's calls in the order a model makes them.

    x [B, L + Lt, C] -> 8-bit projection -> norms of q and k, rotary positions, heads -> router, attention with the gate projected from x -> o

and back to the gradients of x and of all weights.  The projection's three products (forward, dX, dW) run on e4m3 values with a scale for each 128 of
them: weights are quantised once per update in 128 x 128 blocks (both forms), hidden states and gradients as they come, along the dimension that is
summed over.  Master weights stay with the caller.  torch is used for memory, and with text behind the videos of a batch to copy
the video rows next to one another, as the gate's calls take them.

In front of it, Vsa2ResidualNorm: the residual stream with a branch added, and its norm, which is x:

    h = residual + dropout(branch) -> x = norm(h), in bf16 for the gate and in 8 bits for the projection

A layer that only serves can take its projection in whole numbers (projection="int8"): no backward, weights and hidden states with a scale a row.
"""
from __future__ import annotations

from . import binding as vb


class Vsa2ResidualNorm:
    """rows: tokens of a call, batch and all; hidden: channels; p: share of the branch's elements that a training forward drops; seed: of the masks (norms
    with one seed drop the same elements: the norms of a model, and its replicas on other data, need one each); projection: what the 8-bit form of the hidden states is for, as Vsa2Layer's.

    forward gives the stream h, its norm x in bf16, and x's 8-bit form; it keeps what backward needs until the next forward.  h and the weight are kept as they are, not copied: backward
    refuses where torch has changed one of them since.  rng (int64 [2] on the device: seed, offset) is counted on by every forward that drops: a captured step draws anew at each replay.
    backward forms the mask again from what its own forward drew with, whatever rng has become."""

    def __init__(self, rows, hidden, p=0.0, eps=1e-6, seed=0, projection="fp8", device="cuda"):
        import torch
        if projection not in ("fp8", "int8"):
            raise ValueError("projection is fp8 or int8")
        if not 0.0 <= p < 1.0:
            raise ValueError("p is a share of the branch's elements: 0 <= p < 1")
        self.torch, self.rows, self.hidden, self.p, self.eps, self.device = torch, rows, hidden, p, eps, torch.device(device)
        self.form = vb.Int8 if projection == "int8" else vb.Fp8
        self.rng = torch.tensor([seed, 0], dtype=torch.int64, device=device)
        self.next = torch.tensor([0, 1], dtype=torch.int64, device=device)
        self.ws = torch.empty(max(256, vb.vsa2_residual_norm_bwd_workspace_bytes(rows, hidden)), dtype=torch.uint8, device=device)
        self.weight = None
        self.saved, self.kept = None, ()

    def set_weights(self, weight):
        """weight: fp32 [hidden], or None: ones."""
        if weight is not None and (tuple(weight.shape) != (self.hidden,) or weight.dtype != self.torch.float32 or not weight.is_cuda or not weight.is_contiguous()):
            raise ValueError(f"expected the norm's weights as a contiguous CUDA tensor ({self.hidden},) in fp32")
        self.weight = weight

    def _rows(self, t, what):
        """[.., hidden] as the calls' matrix; its type is theirs to look at."""
        if t.shape[-1] != self.hidden or t.numel() != self.rows * self.hidden or not t.is_contiguous():
            raise ValueError(f"expected {what} as a contiguous tensor of {self.rows} rows of {self.hidden} channels, not {tuple(t.shape)}")
        return t.view(self.rows, self.hidden)

    def forward(self, branch, residual, training=True):
        """branch, residual [.., hidden], each bf16 or fp32 -> (h of residual's type, x in bf16, both of residual's shape, x's 8-bit form [rows, hidden])."""
        torch = self.torch
        drops = self.p if training else 0.0
        rng = self.rng + self.next if drops else None      # (a copy of this forward's own)
        h = torch.empty_like(residual)
        x = torch.empty(residual.shape, dtype=torch.bfloat16, device=self.device)
        x8 = self.form.empty(self.rows, self.hidden, self.device)
        vb.vsa2_residual_norm_fwd(self._rows(branch, "the branch"), self._rows(residual, "the residual"), self.weight, eps=self.eps, h=h.view(self.rows, self.hidden), y=x.view(self.rows, self.hidden),
                                  **{"y_int8" if self.form is vb.Int8 else "y_fp8": x8}, p=drops, rng=rng)
        if drops:
            self.rng.copy_(rng)      # (a call that was refused has not counted)
        self.saved, self.kept = (h, branch.shape, branch.dtype, drops, rng, self.weight), self._versions(h)
        return h, x, x8

    def _versions(self, h):
        """torch's counters of changes in place."""
        return tuple(None if t is None or t.is_inference() else t._version for t in (h, self.weight))

    def backward(self, dx, dh=None):
        """Gradients of x (bf16 or fp32) and, where something else reads the stream, of h -> dict of d_residual, d_branch (each of its input's shape and type) and, in fp32, d_weight."""
        if self.saved is None:
            raise RuntimeError("backward without a forward before it")
        h, branch_shape, branch_type, drops, rng, weight = self.saved
        if weight is not self.weight or self._versions(h) != self.kept:
            raise RuntimeError("changed between forward and backward: the stream, or the norm's weights")
        torch = self.torch
        d_residual, d_weight = torch.empty_like(h), torch.empty(self.hidden, dtype=torch.float32, device=self.device)
        d_branch = torch.empty(branch_shape, dtype=branch_type, device=self.device) if drops or branch_type != h.dtype else None
        vb.vsa2_residual_norm_bwd(h.view(self.rows, self.hidden), self._rows(dx, "the gradient of x"), None if dh is None else self._rows(dh, "the gradient of h"), self.weight, eps=self.eps,
                                  d_residual=d_residual.view(self.rows, self.hidden), dx=None if d_branch is None else d_branch.view(self.rows, self.hidden), d_weight=d_weight, workspace=self.ws,
                                  p=drops, rng=rng)
        if d_branch is None:
            d_branch = d_residual if branch_shape == h.shape else d_residual.view(branch_shape)
        return {"d_residual": d_residual, "d_branch": d_branch, "d_weight": d_weight}


class Vsa2Layer:
    """params: the attention's problem (make_params; out_dtype BF16); hidden: channels of x; rope_channels: channels of a head that turn with (t, h, w).

    set_weights takes w_qkv [(Hq + 2 Hkv) D, C] bf16 or fp32 (rows: q's heads, k's, v's), w_g [C, Hq] bf16 and the norms' weights fp32 [D] (None: ones); forward keeps what
    backward needs until the next forward (with an int8 projection, which has none, nothing).  x, o and the weights of the gate and of the norms are kept as they are, not copied: they, and the weights that were set, have to stay until
    backward returns.  It refuses where torch or set_weights has changed one of them since (what other kernels write into them it cannot see)."""

    def __init__(self, params, hidden, rope_channels, theta=1e4, scale=1.0, layout=vb.ROPE_PAIRS, eps=1e-6, device="cuda", projection="fp8"):
        import torch
        if params.out_dtype != vb.BF16:
            raise ValueError("the layer's attention gives bf16 (out_dtype BF16)")
        if projection not in ("fp8", "int8"):
            raise ValueError("projection is fp8 or int8")
        self.torch, self.p, self.hidden, self.eps, self.device = torch, params, hidden, eps, torch.device(device)
        p = params
        self.rope = vb.vsa2_rope_plan(p.head_dim, rope_channels, theta=theta, scale=scale, layout=layout)
        self.attn = vb.Vsa2Attention(p, device)
        self.grid, self.tokens = (p.grid_t, p.grid_h, p.grid_w), int(self.attn.sizes.tokens_per_head)
        self.rows, self.width = p.batch * self.tokens, (p.heads_q + 2 * p.heads_kv) * p.head_dim
        self.int8 = projection == "int8"
        if self.int8:
            self.w, self.w_t = vb.Int8.empty(self.width, hidden, device), None
            need = vb.vsa2_int8_matmul_workspace_bytes(self.rows, self.width, hidden)
        else:
            self.w, self.w_t = vb.Fp8.empty(self.width, hidden, device), vb.Fp8.empty(hidden, self.width, device)
            need = max(vb.vsa2_fp8_matmul_workspace_bytes(*s) for s in ((self.rows, self.width, hidden), (self.rows, hidden, self.width),
                                                                        (self.width, hidden, self.rows)))
        self.ws_matmul = torch.empty(need, dtype=torch.uint8, device=device)
        self.ws_matmul[:256].zero_()      # status block
        self.ws_qkv = torch.empty(vb.vsa2_qkv_bwd_workspace_bytes(p.head_dim), dtype=torch.uint8, device=device)
        self.ws_gate = torch.empty(max(256, vb.vsa2_gate_bwd_workspace_bytes(p, hidden)), dtype=torch.uint8, device=device)
        self.w_g = self.q_weight = self.k_weight = None
        self.saved, self.kept, self.updates = None, (), 0

    def _expect(self, t, what, shape, dtype):
        """The attention and the gate get plain addresses; sizes and types are the layer's."""
        if tuple(t.shape) != shape or t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"expected {what} as a contiguous CUDA tensor {shape} in {dtype}, not {tuple(t.shape)} in {t.dtype}")

    def set_weights(self, w_qkv, w_g, q_weight, k_weight):
        self._expect(w_g, "the gate's weights", (self.hidden, self.p.heads_q), self.torch.bfloat16)
        for w in (q_weight, k_weight):
            if w is not None:
                self._expect(w, "a norm's weights", (self.p.head_dim,), self.torch.float32)
        self.updates += 1
        if self.int8:
            vb.vsa2_int8_quantize(w_qkv, self.w)
        else:
            vb.vsa2_fp8_quantize(w_qkv, self.w, self.w_t, squares=True)
        self.w_g, self.q_weight, self.k_weight = w_g, q_weight, k_weight

    def _heads(self, packed):
        """q, k, v as [B, heads, tokens, D] views of the projection's rows."""
        p = self.p
        v = packed.view(p.batch, self.tokens, p.heads_q + 2 * p.heads_kv, p.head_dim).transpose(1, 2)
        return v[:, :p.heads_q], v[:, p.heads_q:p.heads_q + p.heads_kv], v[:, p.heads_q + p.heads_kv:]

    def _empty(self, *shape, dtype=None):
        return self.torch.empty(*shape, dtype=dtype or self.torch.bfloat16, device=self.device)

    def forward(self, x, x8=None):
        """x [B, L + Lt, C] bf16, contiguous -> o [B, Hq, L + Lt, D] bf16.  x8: x's 8-bit form [B (L + Lt), C] (Fp8, or Int8 for an int8 projection) where the norm has made it."""
        p, torch = self.p, self.torch
        self._expect(x, "hidden states", (p.batch, self.tokens, self.hidden), torch.bfloat16)
        if self.updates == 0:
            raise RuntimeError("forward before set_weights")
        form, quantize, product = (vb.Int8, vb.vsa2_int8_quantize, vb.vsa2_int8_matmul) if self.int8 else (vb.Fp8, vb.vsa2_fp8_quantize, vb.vsa2_fp8_matmul)
        if x8 is None:
            x8 = form.empty(self.rows, self.hidden, self.device)
            quantize(x.view(self.rows, self.hidden), x8)
        elif not isinstance(x8, form) or x8.shape != (self.rows, self.hidden):
            raise ValueError(f"expected the 8-bit form of x as {form.__name__} of {self.rows} rows of {self.hidden} channels")
        packed = self._empty(self.rows, self.width)
        product(x8, self.w, packed, self.ws_matmul)
        q, k, v = (self._empty(p.batch, h, self.tokens, p.head_dim) for h in (p.heads_q, p.heads_kv, p.heads_kv))
        vb.vsa2_qkv_fwd(self.rope, self._heads(packed), (q, k, v), self.q_weight, self.k_weight, eps=self.eps, grid=self.grid)
        video = x[:, :self.attn.sizes.seq_len].contiguous()
        gate = self._empty(p.batch, p.heads_q, self.attn.sizes.seq_len, dtype=torch.float32)
        vb.vsa2_gate_fwd(p, self.hidden, video, self.w_g, gate)
        self.attn.route(q, k)
        o, lse = self.attn.forward(q, k, v, gate)
        if not self.int8:      # (no backward: nothing to keep)
            self.saved = (x, video, packed, q, k, v, gate, o, lse)
            self.kept = self._versions(x, o)
        return o

    def _versions(self, x, o):
        """What backward needs unchanged, as it is now: the number of updates, and torch's counters of changes in place."""
        return (self.updates, *(None if t is None or t.is_inference() else t._version for t in (x, o, self.w_g, self.q_weight, self.k_weight)))

    def backward(self, d_o):
        """d_o [B, Hq, L + Lt, D] bf16 -> dict of dx [B, L + Lt, C] bf16 and, in fp32, dw_qkv, dw_g, dq_weight, dk_weight."""
        p, torch = self.p, self.torch
        if self.int8:
            raise RuntimeError("an int8 projection has no backward")
        if self.saved is None:
            raise RuntimeError("backward without a forward before it")
        x, video, packed, q, k, v, gate, o, lse = self.saved
        now = self._versions(x, o)
        if now != self.kept:
            names = ("the weights (set_weights)", "x", "o", "w_g", "q_weight", "k_weight")
            raise RuntimeError(f"changed between forward and backward: {', '.join(n for n, a, b in zip(names, now, self.kept) if a != b)}")
        self._expect(d_o, "the output's gradient", tuple(o.shape), torch.bfloat16)
        dq, dk, dv, dgate = self.attn.backward(q, k, v, gate, o, lse, d_o)
        d_packed = torch.empty_like(packed)
        dqw, dkw = (self._empty(p.head_dim, dtype=torch.float32) for _ in range(2))
        vb.vsa2_qkv_bwd(self.rope, self._heads(packed), (dq, dk, dv), self._heads(d_packed), self.q_weight, self.k_weight, dqw, dkw, self.ws_qkv,
                        eps=self.eps, grid=self.grid)
        g, g_t, x_t = (vb.Fp8.empty(*s, self.device) for s in ((self.rows, self.width), (self.width, self.rows), (self.hidden, self.rows)))
        vb.vsa2_fp8_quantize(d_packed, g, g_t)
        vb.vsa2_fp8_quantize(x.view(self.rows, self.hidden), None, x_t)
        dx = self._empty(p.batch, self.tokens, self.hidden)
        vb.vsa2_fp8_matmul(g, self.w_t, dx.view(self.rows, self.hidden), self.ws_matmul)
        dw = self._empty(self.width, self.hidden, dtype=torch.float32)
        vb.vsa2_fp8_matmul(g_t, x_t, dw, self.ws_matmul)
        dw_g = self._empty(self.hidden, p.heads_q, dtype=torch.float32)
        vb.vsa2_gate_bwd_add(p, self.hidden, video, self.w_g, gate, dgate, dw_g, dx, self.ws_gate)
        return {"dx": dx, "dw_qkv": dw, "dw_g": dw_g, "dq_weight": dqw, "dk_weight": dkw}

    def check_status(self):
        self.attn.check_status()
        code = vb.vsa2_device_status(self.ws_matmul)
        if code != vb.OK:
            raise vb.Vsa2Error(code, "device status after the projection")
