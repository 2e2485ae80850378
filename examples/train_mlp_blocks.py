"""Trains a few residual MLP blocks on a fixed random regression task, with the GEMMs that carry gradients cut into
sub-GEMM tasks for simulated devices and everything else done by the operators around them:

    forward    rmsnorm (residual added, statistics kept)  ->  linear with bias and GELU, pre-activation kept
               ->  linear with bias, residual for the next block's norm
    backward   planned dgrad + wgrad of the second product  ->  act_backward (dz, bias gradient)
               ->  planned dgrad + wgrad of the first  ->  rmsnorm_backward (joins the residual's gradient)
    update     AdamW over all tensors in one launch, straight from the planned GEMMs' fp32 results; its bf16 copies
               are the next step's operands

    python examples/train_mlp_blocks.py [--steps 60] [--bits 8]
"""
from __future__ import annotations

import argparse
import os
import sys
from types import SimpleNamespace

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import cleave_inputs as ci  # noqa: E402
import paper_2512_22142_b200 as cl  # noqa: E402

DEV = "cuda"


class PlannedGemms:
    """One level of GEMMs, cut into tasks over `devices`; `run` leaves their fp32 results in `C`."""

    def __init__(self, shapes, devices):
        self.gemms = [SimpleNamespace(M=m, N=n, K=k, transA=ta, transB=tb, lda=m if ta else k, ldb=k if tb else n, level=0)
                      for m, n, k, ta, tb in shapes]
        self.plan = cl.plan(self.gemms, devices)
        self.arena = torch.empty(max(1, self.plan.arena_elems), device=DEV)
        self.C = [torch.empty(g.M, g.N, device=DEV) for g in self.gemms]

    def run(self, A, B):
        self.plan.exec_fused(A, B, self.arena, self.C)
        self.plan.assemble(self.arena, self.C)
        return self.C


class Block:
    """y = rmsnorm(h) ; out = gelu(y W1 + b1) W2 + b2, added to h by the next norm."""

    def __init__(self, tokens, d, ffn, devices, gen):
        def master(*shape, scale):
            return torch.randn(*shape, generator=gen, device=DEV) * scale
        self.params = {"norm": torch.ones(d, device=DEV), "W1": master(d, ffn, scale=d ** -0.5), "b1": torch.zeros(ffn, device=DEV),
                       "W2": master(ffn, d, scale=ffn ** -0.5), "b2": torch.zeros(d, device=DEV)}
        self.copies = {k: v.to(torch.bfloat16) for k, v in self.params.items()}
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        self.h, self.rstd = torch.empty(tokens, d, device=DEV), torch.empty(tokens, device=DEV)
        self.y, self.z, self.a, self.out = bf(tokens, d), bf(tokens, ffn), bf(tokens, ffn), bf(tokens, d)
        self.dz, self.dh = bf(tokens, ffn), torch.empty(tokens, d, device=DEV)
        self.second = PlannedGemms([(tokens, ffn, d, 0, 1), (ffn, d, tokens, 1, 0)], devices)     # dout W2^T, a^T dout
        self.first = PlannedGemms([(tokens, d, ffn, 0, 1), (d, ffn, tokens, 1, 0)], devices)      # dz W1^T, y^T dz
        self.grads = {"norm": torch.empty(d, device=DEV), "W1": self.first.C[1], "b1": torch.empty(ffn, device=DEV), "W2": self.second.C[1],
                      "b2": torch.empty(d, device=DEV)}

    def forward(self, x, residual):
        """x: the block before's output (bf16); residual: its h (fp32)."""
        w = self.copies
        cl.rmsnorm(x, self.params["norm"], self.y, residual=residual, h=self.h, rstd=self.rstd)
        cl.linear(self.y, w["W1"], self.a, bias=self.params["b1"], act="gelu_tanh", z=self.z)
        cl.linear(self.a, w["W2"], self.out, bias=self.params["b2"])
        return self.out, self.h

    def backward(self, dout, dh):
        """dout: gradient of out (bf16); dh: what reaches h past this block (fp32).  Returns the gradient of h."""
        w = self.copies
        da, _ = self.second.run([dout, self.a], [w["W2"], dout])
        cl.act_backward(dout, None, dbias=self.grads["b2"])
        cl.act_backward(da, self.z, self.dz, act="gelu_tanh", dbias=self.grads["b1"])
        dy, _ = self.first.run([self.dz, self.y], [w["W1"], self.dz])
        cl.rmsnorm_backward(dy, self.h, self.params["norm"], self.rstd, self.dh, self.grads["norm"], dres=dh)
        return self.dh


def train(steps=60, bits=8, tokens=1024, d=256, ffn=768, blocks=2, n_devices=24, lr=2e-3, seed=0):
    """Losses of `steps` steps."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    devices = ci.make_devices(n_devices, 64 * ci.MB, ci.GB, seed)
    stack = [Block(tokens, d, ffn, devices, gen) for _ in range(blocks)]
    x = torch.randn(tokens, d, generator=gen, device=DEV)
    target = torch.tanh(x @ torch.randn(d, d, generator=gen, device=DEV) * d ** -0.5).roll(1, dims=1)
    zero = torch.zeros(tokens, d, dtype=torch.bfloat16, device=DEV)

    names = list(stack[0].params)
    flat = lambda attr: [getattr(b, attr)[k].view(-1) for b in stack for k in names]  # noqa: E731
    params = flat("params")
    scales = {}
    if bits == 8:
        state = [[torch.zeros(p.numel(), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for p in params] for _ in range(2)]
        scales = {k: [torch.zeros(-(-p.numel() // 256), device=DEV) for p in params] for k in ("m_scales", "v_scales")}
    else:
        state = [[torch.zeros_like(p) for p in params] for _ in range(2)]
    opt = cl.AdamW(params, flat("grads"), state[0], state[1], copies=flat("copies"),
                   weight_decay=[0.01 if k in ("W1", "W2") else 0.0 for _ in stack for k in names], **scales)
    losses = []
    for step in range(1, steps + 1):
        out, h = zero, x
        for b in stack:
            out, h = b.forward(out, h)
        error = h + out.float() - target
        losses.append(error.square().mean())
        dh = error * (2.0 / error.numel())
        for b in reversed(stack):
            dh = b.backward(dh.to(torch.bfloat16), dh)
        opt.step(step=step, lr=lr, seed=seed)
    assert cl.linear_status() == 0
    for b in stack:
        b.first.plan.check_status()
        b.second.plan.check_status()
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    args = ap.parse_args()
    for i, v in enumerate(train(args.steps, args.bits)):
        if i % 10 == 0 or i == args.steps - 1:
            print(f"step {i + 1:4d}  loss {v:.5f}")
