"""One self-attention layer from its hidden states on: the library's calls in the order a model makes them.

    x [B, L + Lt, C] -> 8-bit projection -> norms of q and k, rotary positions, heads -> router, attention with the gate projected from x -> o

and back to the gradients of x and of all weights.  The projection's three products (forward, dX, dW) run on e4m3 values with a scale for each 128 of
them: weights are quantised once per update in 128 x 128 blocks (both forms), hidden states and gradients as they come, along the dimension that is
summed over.  Master weights stay with the caller.  torch is used for memory, and with text behind the videos of a batch to copy
the video rows next to one another, as the gate's calls take them.
"""
from __future__ import annotations

from . import binding as vb


class Vsa2Layer:
    """params: the attention's problem (make_params; out_dtype BF16); hidden: channels of x; rope_channels: channels of a head that turn with (t, h, w).

    set_weights takes w_qkv [(Hq + 2 Hkv) D, C] bf16 or fp32 (rows: q's heads, k's, v's), w_g [C, Hq] bf16 and the norms' weights fp32 [D] (None: ones); forward keeps what
    backward needs until the next forward.  x, o and the weights of the gate and of the norms are kept as they are, not copied: they, and the weights that were set, have to stay until
    backward returns.  It refuses where torch or set_weights has changed one of them since (what other kernels write into them it cannot see)."""

    def __init__(self, params, hidden, rope_channels, theta=1e4, scale=1.0, layout=vb.ROPE_PAIRS, eps=1e-6, device="cuda"):
        import torch
        if params.out_dtype != vb.BF16:
            raise ValueError("the layer's attention gives bf16 (out_dtype BF16)")
        self.torch, self.p, self.hidden, self.eps, self.device = torch, params, hidden, eps, torch.device(device)
        p = params
        self.rope = vb.vsa2_rope_plan(p.head_dim, rope_channels, theta=theta, scale=scale, layout=layout)
        self.attn = vb.Vsa2Attention(p, device)
        self.grid, self.tokens = (p.grid_t, p.grid_h, p.grid_w), int(self.attn.sizes.tokens_per_head)
        self.rows, self.width = p.batch * self.tokens, (p.heads_q + 2 * p.heads_kv) * p.head_dim
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
        vb.vsa2_fp8_quantize(w_qkv, self.w, self.w_t, squares=True)
        self.w_g, self.q_weight, self.k_weight = w_g, q_weight, k_weight

    def _heads(self, packed):
        """q, k, v as [B, heads, tokens, D] views of the projection's rows."""
        p = self.p
        v = packed.view(p.batch, self.tokens, p.heads_q + 2 * p.heads_kv, p.head_dim).transpose(1, 2)
        return v[:, :p.heads_q], v[:, p.heads_q:p.heads_q + p.heads_kv], v[:, p.heads_q + p.heads_kv:]

    def _empty(self, *shape, dtype=None):
        return self.torch.empty(*shape, dtype=dtype or self.torch.bfloat16, device=self.device)

    def forward(self, x):
        """x [B, L + Lt, C] bf16, contiguous -> o [B, Hq, L + Lt, D] bf16."""
        p, torch = self.p, self.torch
        self._expect(x, "hidden states", (p.batch, self.tokens, self.hidden), torch.bfloat16)
        if self.updates == 0:
            raise RuntimeError("forward before set_weights")
        a = vb.Fp8.empty(self.rows, self.hidden, self.device)
        vb.vsa2_fp8_quantize(x.view(self.rows, self.hidden), a)
        packed = self._empty(self.rows, self.width)
        vb.vsa2_fp8_matmul(a, self.w, packed, self.ws_matmul)
        q, k, v = (self._empty(p.batch, h, self.tokens, p.head_dim) for h in (p.heads_q, p.heads_kv, p.heads_kv))
        vb.vsa2_qkv_fwd(self.rope, self._heads(packed), (q, k, v), self.q_weight, self.k_weight, eps=self.eps, grid=self.grid)
        video = x[:, :self.attn.sizes.seq_len].contiguous()
        gate = self._empty(p.batch, p.heads_q, self.attn.sizes.seq_len, dtype=torch.float32)
        vb.vsa2_gate_fwd(p, self.hidden, video, self.w_g, gate)
        self.attn.route(q, k)
        o, lse = self.attn.forward(q, k, v, gate)
        self.saved = (x, video, packed, q, k, v, gate, o, lse)
        self.kept = self._versions(x, o)
        return o

    def _versions(self, x, o):
        """What backward needs unchanged, as it is now: the number of updates, and torch's counters of changes in place."""
        return (self.updates, *(None if t is None or t.is_inference() else t._version for t in (x, o, self.w_g, self.q_weight, self.k_weight)))

    def backward(self, d_o):
        """d_o [B, Hq, L + Lt, D] bf16 -> dict of dx [B, L + Lt, C] bf16 and, in fp32, dw_qkv, dw_g, dq_weight, dk_weight."""
        p, torch = self.p, self.torch
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
