"""One OpenLM transformer block on the GPU (forward and backward).

The paper's models are OpenLM transformers (Sec. 3.1; Table "openlm1b":
hidden dimension 2048, 24 layers, 16 heads, 1,439,893,504 parameters) with
RoPE (Sec. 3, "Positional encoding").  The block, with the readings that
reproduce that parameter count exactly (50,432-token vocabulary, untied
embeddings):

    a = LayerNorm_1(x);  q, k, v = a W_qkv   (H heads of D = d / H)
    h = x + Attention(RoPE(q), RoPE(k), v) W_o
    m = LayerNorm_2(h);  y = h + (silu(m W_1) * (m W_3)) W_2

LayerNorms have weight and bias, projections have none, the SwiGLU width is
5632 at d = 2048.  Every step runs in this library's HIP kernels: the
projections and the MLP products in its bf16 GEMM (the residual additions
and the SwiGLU, forward and backward, in the GEMM epilogue; products that
share an input or are summed run as one launch), the LayerNorms in their own
kernels, RoPE and attention in the attention kernels; the backward is written out
step by step (one autograd node for the whole block).  The block exists to
place the attention hot path in a full layer step: its time as a share of
the step, and the step time's growth with the sequence length at a fixed
token budget.

With ``checkpoint_bits=8`` the block keeps five of its activations between
forward and backward as int8 codes with a scale per token instead of bf16: the
outputs of the norms, the two gate products and the gated value (of the 1B
block's 66.6 KB a token 45.6 are left; with what the passes themselves need,
91 of 101 at the peak).  A step of 65,536 tokens takes 4 to 7% longer for it.
Without a backward no codes are formed.  The forward is the same; the backward
forms the weight gradients from the codes and the gate's gradient from the
restored values, so gradients carry the codes' rounding, at most half a step
of a token's largest value / 127.  The width of the SwiGLU is then at most
16384.

Shapes: B*L, d and the SwiGLU width multiples of 256, d in
{512, 1024, 2048}, d / H in {64, 128}.
"""
from __future__ import annotations

import torch

from . import block_ops as ops
from .attention import _doclens, backward_rope, forward_rope

LN_EPS = 1e-5
OPENLM_1B = dict(d=2048, H=16, hidden=5632)


class _BlockFunction(torch.autograd.Function):
    """Forward and backward of one block on x [T, d] (T = B * L tokens)."""

    @staticmethod
    def forward(ctx, x, ln1_w, ln1_b, w_qkv, w_o, ln2_w, ln2_b, w_1, w_3, w_2, shape, base,
                docs, doc_pos, bits):
        B, L, H, D = shape
        d = H * D
        codes = bits == 8 and any(ctx.needs_input_grad)
        kept = []

        def keep(act):  # the last use of an activation: its codes take its place
            kept.extend(ops.quantize(act) if codes else (act,))

        a, mean1, rstd1 = ops.layer_norm(x, ln1_w, ln1_b, LN_EPS)
        q, k, v = ops.gemm_group(a, [w_qkv[:, i * d:(i + 1) * d] for i in range(3)])
        keep(a)
        del a
        o, lse, qr, kr = forward_rope(q.view(B, L, H, D), k.view(B, L, H, D),
                                      v.view(B, L, H, D), base, True, docs, doc_pos)
        o2 = o.view(B * L, d)
        h = ops.gemm(o2, w_o, residual=x)
        m, mean2, rstd2 = ops.layer_norm(h, ln2_w, ln2_b, LN_EPS)
        u1, u3, g = ops.gemm_swiglu(m, w_1, w_3)
        keep(m)
        del m
        keep(u1)
        del u1
        keep(u3)
        del u3
        y = ops.gemm(g, w_2, residual=h)
        keep(g)
        ctx.save_for_backward(x, ln1_w, w_qkv, w_o, ln2_w, w_1, w_3, w_2, mean1, rstd1, qr, kr, v,
                              o, lse, h, mean2, rstd2, *kept)
        ctx.cfg = (shape, base, docs, doc_pos, bits)
        return y

    @staticmethod
    def backward(ctx, dy):
        (x, ln1_w, w_qkv, w_o, ln2_w, w_1, w_3, w_2, mean1, rstd1, qr, kr, v, o, lse, h, mean2,
         rstd2, *kept) = ctx.saved_tensors
        (B, L, H, D), base, docs, doc_pos, bits = ctx.cfg
        d = H * D
        dy = dy.contiguous()
        if bits == 8:
            a, m, u1, u3, g = zip(kept[::2], kept[1::2])

            def weight_grads(act, dys, outs=None):
                return ops.gemm_int8_wgrad_group(*act, dys, outs=outs)
        else:
            a, m, u1, u3, g = kept

            def weight_grads(act, dys, outs=None):
                return ops.gemm_group(act, dys, trans_a=True, outs=outs)
        # MLP: y = h + swiglu(m W1, m W3) W2 (each restored activation only as
        # long as it is read: the weight gradients hold one too)
        dw_2, = weight_grads(g, [dy])
        if bits == 8:
            u1, u3 = ops.dequantize(*u1), ops.dequantize(*u3)
        du1, du3 = ops.gemm_swiglu_backward(dy, w_2, u1, u3)
        del u1, u3
        dm = ops.gemm_sum([du1, du3], [w_1, w_3], trans_b=True)
        dw_1, dw_3 = weight_grads(m, [du1, du3])
        del du1, du3
        dh, dln2_w, dln2_b = ops.layer_norm_backward(h, ln2_w, mean2, rstd2, dm, dres=dy)
        # attention: h = x + attn(RoPE(q), RoPE(k), v) Wo
        do = ops.gemm(dh, w_o, trans_b=True)
        dw_o = ops.gemm(o.view(B * L, d), dh, trans_a=True)
        dq, dk, dv = backward_rope(qr, kr, v.view(B, L, H, D), o, lse, do.view(B, L, H, D),
                                   base, True, docs, doc_pos)
        grads = [t.view(B * L, d) for t in (dq, dk, dv)]
        columns = [slice(i * d, (i + 1) * d) for i in range(3)]
        da = ops.gemm_sum(grads, [w_qkv[:, c] for c in columns], trans_b=True)
        dw_qkv = torch.empty_like(w_qkv)
        weight_grads(a, grads, [dw_qkv[:, c] for c in columns])
        dx, dln1_w, dln1_b = ops.layer_norm_backward(x, ln1_w, mean1, rstd1, da, dres=dh)
        return (dx, dln1_w, dln1_b, dw_qkv, dw_o, dln2_w, dln2_b, dw_1, dw_3, dw_2,
                None, None, None, None, None)


class OpenLMBlock(torch.nn.Module):
    def __init__(self, d: int = 2048, H: int = 16, hidden: int = 5632, rope_base=100000.0,
                 device="cuda", dtype=torch.bfloat16, seed: int = 0, init_scale: float = 0.02,
                 checkpoint_bits: int = 16):
        super().__init__()
        if d % H:
            raise ValueError("d must be a multiple of H")
        if checkpoint_bits not in (8, 16):
            raise ValueError(f"checkpoint_bits must be 8 or 16 (got {checkpoint_bits})")
        if checkpoint_bits == 8 and hidden > ops.MAX_ROW:
            raise ValueError(f"checkpoint_bits=8 takes a width of at most {ops.MAX_ROW} "
                             f"(got {hidden})")
        self.checkpoint_bits = checkpoint_bits
        self.d, self.H, self.D, self.hidden = d, H, d // H, hidden
        self.rope_base = rope_base
        g = torch.Generator(device="cpu").manual_seed(seed)

        def mat(*shape):
            w = torch.randn(*shape, generator=g) * init_scale
            return torch.nn.Parameter(w.to(device=device, dtype=dtype))

        def vec(fill):
            return torch.nn.Parameter(torch.full((d,), fill, device=device, dtype=dtype))

        # weights map rows by right multiplication: x [T, in] @ W [in, out]
        self.ln1_w, self.ln1_b = vec(1.0), vec(0.0)
        self.w_qkv = mat(d, 3 * d)
        self.w_o = mat(d, d)
        self.ln2_w, self.ln2_b = vec(1.0), vec(0.0)
        self.w_1 = mat(d, hidden)
        self.w_3 = mat(d, hidden)
        self.w_2 = mat(hidden, d)

    def weights(self) -> dict:
        return {n: p for n, p in self.named_parameters()}

    def forward(self, x, cu_doclens=None, doc_positions: bool = False):
        B, L, d = x.shape
        docs = _doclens(cu_doclens, B, L, x.device)
        # without a backward nothing is kept, so no codes are formed
        bits = self.checkpoint_bits if torch.is_grad_enabled() else 16
        y = _BlockFunction.apply(x.reshape(B * L, d), self.ln1_w, self.ln1_b, self.w_qkv,
                                 self.w_o, self.ln2_w, self.ln2_b, self.w_1, self.w_3, self.w_2,
                                 (B, L, self.H, self.D), self.rope_base, docs, doc_positions,
                                 bits)
        return y.view(B, L, d)

    def gemm_flops(self, tokens: int) -> int:
        """Forward FLOPs of the projections and the MLP (backward: twice this)."""
        d, h = self.d, self.hidden
        return 2 * tokens * (4 * d * d + 3 * d * h)
