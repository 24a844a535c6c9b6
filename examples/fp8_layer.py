#!/usr/bin/env python3
"""A Llama-shaped transformer layer with 8-bit linear layers: training step and decoding of single tokens.

The residual stream is carried as two tensors, `x` (what the last block put out) and `res` (the stream it is to be added to): the
addition is part of the next norm, and its gradient of that norm's backward.  Per linear layer y = x W^T the products are
    y = x_r W_r^T,    dx = dy_r W_c^T,    dW += dy_c x_c^T
over operands by rows (r) and by columns (c); weights are laid out in both ways once per optimizer step, activations as
e4m3 and gradients as e5m2 when they arise.  What the backward needs of an activation is kept in 8 bits.

    python examples/fp8_layer.py                       # 8B-shaped layer, 8192 tokens
    python examples/fp8_layer.py --tokens 4093 --steps 5
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_27089_amd import binding as sp  # noqa: E402

E5M2 = torch.float8_e5m2
EPS = 1e-5


def rope_tables(n, D, device, base=500000.0):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    return angle.cos().float().to(device), angle.sin().float().to(device)


class Linear:
    """A weight [F, C] bf16, its operands by rows and by columns, and its gradient in fp32."""

    def __init__(self, weight, training):
        self.weight = weight
        self.grad = torch.zeros(weight.shape, dtype=torch.float32, device=weight.device) if training else None
        self.q, self.q_scale, self.qt, self.qt_scale = sp.sp_fp8_quant(weight, cols=training)

    def forward(self, x, x_scale):
        return sp.sp_fp8_matmul(x, x_scale, self.q, self.q_scale)

    def backward(self, dy, xt, xt_scale):
        """dy [T, F] bf16, xt the operand of x's transpose -> dx [T, C] bf16; adds to the weight's gradient."""
        g, g_scale, gt, gt_scale = sp.sp_fp8_quant(dy, dtype=E5M2, cols=True)
        sp.sp_fp8_matmul(gt, gt_scale, xt, xt_scale, out=self.grad, accumulate=True)
        return sp.sp_fp8_matmul(g, g_scale, self.qt, self.qt_scale)


class Layer:
    def __init__(self, C, Hq, Hkv, D, F, device="cuda", seed=0, training=True):
        g = torch.Generator(device=device).manual_seed(seed)
        draw = lambda rows, cols: (torch.randn(rows, cols, device=device, generator=g) * cols ** -0.5).to(torch.bfloat16)
        self.C, self.Hq, self.Hkv, self.D = C, Hq, Hkv, D
        self.norm1 = (1 + 0.1 * torch.randn(C, device=device, generator=g)).to(torch.bfloat16)
        self.norm2 = (1 + 0.1 * torch.randn(C, device=device, generator=g)).to(torch.bfloat16)
        # the norms' gradients, added up in fp32 over the calls (one call's arrives in bf16)
        self.dnorm1, self.dnorm2 = (torch.zeros(C, dtype=torch.float32, device=device) if training else None for _ in range(2))
        for name, rows, cols in (("wq", Hq * D, C), ("wk", Hkv * D, C), ("wv", Hkv * D, C), ("wo", C, Hq * D),
                                 ("wg", F, C), ("wu", F, C), ("wd", C, F)):
            setattr(self, name, Linear(draw(rows, cols), training))

    def qkv(self, n, n_scale, cos, sin):
        T = n.shape[0]
        q, k, v = (m.forward(n, n_scale).view(T, -1, self.D) for m in (self.wq, self.wk, self.wv))
        sp.sp_rope(q, cos, sin, out=q)
        sp.sp_rope(k, cos, sin, out=k)
        return q, k, v

    def forward(self, x, res, cos, sin):
        """x, res [T, C] (res None for the first layer), one document -> (y, stream [T, C], what the backward needs)."""
        T = x.shape[0]
        h1, n, n_scale, rstd1 = sp.sp_rmsnorm_fp8_fwd(x, self.norm1, EPS, res=res)
        q, k, v = self.qkv(n, n_scale, cos, sin)
        o, lse = sp.sp_attn_fwd(q[None], k[None], v[None])
        o8, o8_scale, ot, ot_scale = sp.sp_fp8_quant(o.view(T, -1), cols=True)
        h2, n, n_scale, rstd2 = sp.sp_rmsnorm_fp8_fwd(self.wo.forward(o8, o8_scale), self.norm2, EPS, res=h1)
        g, u = self.wg.forward(n, n_scale), self.wu.forward(n, n_scale)
        s8, s8_scale, st, st_scale = sp.sp_fp8_quant(sp.sp_swiglu_fwd(g, u), cols=True)
        return self.wd.forward(s8, s8_scale), h2, (h1, rstd1, q, k, v, o, lse, ot, ot_scale, h2, rstd2, g, u, st, st_scale)

    def backward(self, dy, dstream, kept, cos, sin):
        """Gradients of y and of the stream -> the gradient of x and res alike; those of all weights are added to theirs."""
        h1, rstd1, q, k, v, o, lse, ot, ot_scale, h2, rstd2, g, u, st, st_scale = kept
        T = dy.shape[0]
        dg, du = sp.sp_swiglu_bwd(g, u, self.wd.backward(dy, st, st_scale))
        _, _, nt, nt_scale = sp.sp_fp8_quant(h2, rows=False, cols=True, rstd=rstd2, w=self.norm2)
        dn = self.wg.backward(dg, nt, nt_scale).add_(self.wu.backward(du, nt, nt_scale))
        dh, dw = sp.sp_rmsnorm_res_bwd(h2, self.norm2, rstd2, dn, dstream)
        self.dnorm2.add_(dw.float())
        do = self.wo.backward(dh, ot, ot_scale)
        dq, dk, dv = sp.sp_attn_bwd(q[None], k[None], v[None], o, lse, do.view(1, T, self.Hq, self.D))
        for t in (dq[0], dk[0]):
            sp.sp_rope(t, cos, sin, conjugate=True, out=t)
        _, _, nt, nt_scale = sp.sp_fp8_quant(h1, rows=False, cols=True, rstd=rstd1, w=self.norm1)
        dn = self.wq.backward(dq.view(T, -1), nt, nt_scale)
        dn.add_(self.wk.backward(dk.view(T, -1), nt, nt_scale)).add_(self.wv.backward(dv.view(T, -1), nt, nt_scale))
        dh, dw = sp.sp_rmsnorm_res_bwd(h1, self.norm1, rstd1, dn, dh)
        self.dnorm1.add_(dw.float())
        return dh

    def decode(self, x, res, keys, values, at, cos, sin):
        """x, res [n, C]: the tokens at positions at .. at + n - 1 of one sequence; keys, values [positions, Hkv, D] hold the
        earlier ones and receive these -> (y, stream)."""
        n = x.shape[0]
        h1, a, a_scale, _ = sp.sp_rmsnorm_fp8_fwd(x, self.norm1, EPS, res=res)
        q, k, v = self.qkv(a, a_scale, cos[at:at + n], sin[at:at + n])
        keys[at:at + n] = k
        values[at:at + n] = v
        o, _ = sp.sp_attn_block_fwd(q[None], keys[None, :at + n], values[None, :at + n], causal_offset=at)
        a, a_scale, _, _ = sp.sp_fp8_quant(o.view(n, -1))
        h2, a, a_scale, _ = sp.sp_rmsnorm_fp8_fwd(self.wo.forward(a, a_scale), self.norm2, EPS, res=h1)
        a, a_scale, _, _ = sp.sp_fp8_quant(sp.sp_swiglu_fwd(self.wg.forward(a, a_scale), self.wu.forward(a, a_scale)))
        return self.wd.forward(a, a_scale), h2


def milliseconds(run, steps):
    run()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(steps):
        run()
    end.record()
    end.synchronize()
    return begin.elapsed_time(end) / steps


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("tokens", 8192), ("dim", 4096), ("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("ffn", 14336), ("steps", 10)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    T, C, Hq, Hkv, D, F = a.tokens, a.dim, a.heads, a.kv_heads, a.head_dim, a.ffn
    layer = Layer(C, Hq, Hkv, D, F)
    cos, sin = rope_tables(T, D, "cuda")
    x, res, d = (torch.randn(T, C, device="cuda").to(torch.bfloat16) for _ in range(3))
    fwd = milliseconds(lambda: layer.forward(x, res, cos, sin), a.steps)
    kept = layer.forward(x, res, cos, sin)[2]
    bwd = milliseconds(lambda: layer.backward(d, d, kept, cos, sin), a.steps)
    linear = 2.0 * T * C * (2 * (Hq + Hkv) * D + 3 * F)
    attention = 2.0 * T * (T + 1) * D * Hq
    print(f"{T} tokens, {C} wide: forward {fwd:.3f} ms, backward {bwd:.3f} ms, "
          f"{(3 * linear + 3.5 * attention) / (fwd + bwd) / 1e9:.0f} TFLOP/s ({3 * linear / 1e12:.1f} linear, {3.5 * attention / 1e12:.1f} attention)")
    keys, values = (torch.randn(T, Hkv, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    one = milliseconds(lambda: layer.decode(x[-1:], res[-1:], keys, values, T - 1, cos, sin), 10 * a.steps)
    print(f"one token at position {T - 1}: {one * 1e3:.0f} us")


if __name__ == "__main__":
    main()
