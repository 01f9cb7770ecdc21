"""A Llama-shaped gated MLP, y = (silu(x Wg^T) * (x Wu^T)) Wd^T, trained and served on one MI355X with the library's
operators:

  1. Wd is quantized to NVFP4 and stays frozen; Wg and Wu are trained in bfloat16 to take up its error: swiglu_ffn and
     matmul forwards, matmul_grad_input and swiglu_ffn_backward backwards, through torch's autograd.
  2. Wg and Wu are quantized to microscaled FP4, and prompts and single tokens are served with 4-bit weights alone:
     mx_quantize and mx_matmul for the two projections, swiglu, and matmul for the NVFP4 one.

    python examples/gated_mlp.py [--hidden 1024] [--inner 2816] [--tokens 2048] [--steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_07618_amd as nv  # noqa: E402


class GatedBlock(torch.autograd.Function):
    """h = silu(x Wg^T) * (x Wu^T)."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up):
        h, gate, up = nv.swiglu_ffn(x, w_gate, w_up, save=True)
        ctx.save_for_backward(x, w_gate, w_up, gate, up)
        return h

    @staticmethod
    def backward(ctx, dh):
        needs = ctx.needs_input_grad
        return nv.swiglu_ffn_backward(dh.contiguous(), *ctx.saved_tensors, need_x=needs[0], need_w=needs[1] or needs[2])


class FrozenLinear(torch.autograd.Function):
    """y = h W^T through frozen NVFP4 weights (q, scales, S)."""

    @staticmethod
    def forward(ctx, h, q, scales, S, block):
        ctx.save_for_backward(q, scales, S)
        ctx.block = block
        return nv.matmul(h, q, scales, S, block)

    @staticmethod
    def backward(ctx, dy):
        return nv.matmul_grad_input(dy, *ctx.saved_tensors, ctx.block), None, None, None, None


def rel(a, b):
    return ((a.float() - b.float()).norm() / b.float().norm()).item()


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--hidden", type=int, default=1024)
    p.add_argument("--inner", type=int, default=2816)
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--block", type=int, default=16, help="values under one scale of the NVFP4 weights")
    a = p.parse_args(argv)
    dev = torch.device("cuda")
    g = torch.Generator(dev).manual_seed(0)

    def normal(rows, cols, scale):
        return (torch.randn((rows, cols), generator=g, device=dev) * scale).bfloat16()

    w_gate, w_up = (normal(a.inner, a.hidden, a.hidden ** -0.5) for _ in range(2))
    w_down = normal(a.hidden, a.inner, a.inner ** -0.5)
    x = normal(a.tokens, a.hidden, 1.0)
    whole = nv.swiglu_ffn(x, w_gate, w_up)
    target = whole.float() @ w_down.float().t()                  # what the unquantized block gives

    down = nv.quantize(w_down, "scalesweep_mse", block=a.block)
    train = [w.float().requires_grad_() for w in (w_gate, w_up)]  # binary32 masters of the trained weights
    opt = torch.optim.Adam(train, lr=2e-4)
    losses = []
    for _ in range(a.steps):
        h = GatedBlock.apply(x, train[0].bfloat16(), train[1].bfloat16())
        loss = (FrozenLinear.apply(h, *down, a.block).float() - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    print(f"trained through NVFP4 weights: loss {losses[0]:.3e} -> {losses[-1]:.3e}", flush=True)

    w_gate, w_up = (w.detach().bfloat16() for w in train)
    trained = nv.matmul(nv.swiglu_ffn(x, w_gate, w_up), *down, a.block)
    mx_gate, mx_up = nv.mx_quantize(w_gate), nv.mx_quantize(w_up)

    def serve(rows):
        xq = nv.mx_quantize(rows)
        return nv.matmul(nv.swiglu(nv.mx_matmul(xq, mx_gate), nv.mx_matmul(xq, mx_up)), *down, a.block)

    prompt = serve(x)
    tokens = torch.cat([serve(x[i:i + 1]) for i in range(4)])     # as a decoder asks for them
    errors = {"prompt": rel(prompt, trained), "tokens": rel(tokens, trained[:4]), "gate": rel(
        nv.mx_dequant(*mx_gate, cols=a.hidden), w_gate), "down": rel(nv.dequant(*down, block=a.block), w_down)}
    nbytes = sum(t.numel() * t.element_size() for w in (mx_gate, mx_up, down) for t in w)
    print(f"served with 4-bit weights: {nbytes / 2 ** 20:.1f} MiB in place of {a.inner * a.hidden * 6 / 2 ** 20:.1f}; relative "
          + ", ".join(f"{k} {v:.3f}" for k, v in errors.items()), flush=True)
    return losses, errors


if __name__ == "__main__":
    main()
