"""The operators together with planned GEMMs: the example's training loop against the same step written with torch
in fp32, and the two widths of optimizer state against each other."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _torch_losses(steps, tokens, d, ffn, blocks, lr, seed):
    """The same model and task in fp32 with autograd and torch's AdamW."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    layers = []
    for _ in range(blocks):
        W1 = (torch.randn(d, ffn, generator=gen, device="cuda") * d ** -0.5).requires_grad_()
        W2 = (torch.randn(ffn, d, generator=gen, device="cuda") * ffn ** -0.5).requires_grad_()
        rest = [torch.ones(d, device="cuda", requires_grad=True), torch.zeros(ffn, device="cuda", requires_grad=True), torch.zeros(d, device="cuda", requires_grad=True)]
        layers.append((rest[0], W1, rest[1], W2, rest[2]))
    x = torch.randn(tokens, d, generator=gen, device="cuda")
    target = torch.tanh(x @ torch.randn(d, d, generator=gen, device="cuda") * d ** -0.5).roll(1, dims=1)
    opt = torch.optim.AdamW([{"params": [w for n, a, b, c, e in layers for w in (a, c)], "weight_decay": 0.01},
                             {"params": [w for n, a, b, c, e in layers for w in (n, b, e)], "weight_decay": 0.0}], lr=lr, betas=(0.9, 0.999), eps=1e-8)
    losses = []
    for _ in range(steps):
        h = x
        for n, W1, b1, W2, b2 in layers:
            y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-5) * n
            h = h + torch.nn.functional.gelu(y @ W1 + b1, approximate="tanh") @ W2 + b2
        loss = (h - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return losses


def test_training_follows_torch_and_both_state_widths_agree():
    from train_mlp_blocks import train
    size = dict(tokens=512, d=128, ffn=384, blocks=2, lr=2e-3, seed=3)
    want = _torch_losses(40, **size)
    wide, narrow = train(steps=40, bits=32, n_devices=12, **size), train(steps=40, bits=8, n_devices=12, **size)
    assert want[-1] < 0.5 * want[0]                       # the task is learnt at all
    # bf16 operands: half a unit of 2^-8 on every product's inputs, averaged over hundreds of terms a sum; 2 % holds
    # the first step's loss (one forward pass) with room, 5 % the path of 40 steps, 10 % that of 8-bit states
    assert abs(wide[0] / want[0] - 1) < 0.02 and wide[0] == narrow[0]
    assert max(abs(a / b - 1) for a, b in zip(wide, want)) < 0.05
    assert max(abs(a / b - 1) for a, b in zip(narrow, want)) < 0.10
