"""Trains a small model of tokens whose table is also its output projection, on a fixed random map from token to next token, with the
GEMMs that carry gradients cut into sub-GEMM tasks for simulated devices and everything else done by the operators around them:

    forward    embedding (rows scaled)  ->  blocks: layernorm (residual added, statistics kept) -> linear with bias and GELU
               -> linear with bias  ->  layernorm  ->  linear with the table: scores
    loss       token_logprobs of the next tokens, or distill from the best scores of a teacher
    backward   their backward passes  ->  planned dgrad + wgrad of the table  ->  layernorm_backward, act_backward and planned
               dgrad + wgrad through the blocks  ->  embedding_backward, added to what the output projection left
    update     AdamW over all tensors in one launch; its bf16 copies are the next step's operands

    python examples/train_token_model.py [--steps 60] [--teacher]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path[:0] = [os.path.dirname(os.path.abspath(__file__)), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]
import cleave_inputs as ci  # noqa: E402
import paper_2512_22142_b200 as cl  # noqa: E402
from train_mlp_blocks import DEV, PlannedGemms  # noqa: E402

PADDING = -100


def _bf16(*shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device=DEV)


class Norm:
    """y = layernorm(x + residual) weight + bias, and its gradients."""

    def __init__(self, tokens, d):
        self.params = {"w": torch.ones(d, device=DEV), "b": torch.zeros(d, device=DEV)}
        self.grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        self.h, self.mean, self.rstd = torch.empty(tokens, d, device=DEV), torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV)
        self.y, self.dh = _bf16(tokens, d), torch.empty(tokens, d, device=DEV)

    def forward(self, x, residual):
        cl.layernorm(x, self.params["w"], self.params["b"], self.y, residual=residual, h=self.h, mean=self.mean, rstd=self.rstd)
        return self.y, self.h

    def backward(self, dy, dh):
        """dh: the gradient that reaches h past the norm, or None."""
        cl.layernorm_backward(dy, self.h, self.params["w"], self.mean, self.rstd, self.dh, self.grads["w"], self.grads["b"], dres=dh)
        return self.dh


class Block:
    """out = gelu(layernorm(h) W1 + b1) W2 + b2, added to h by the next norm."""

    def __init__(self, tokens, d, ffn, devices, gen):
        self.norm = Norm(tokens, d)
        self.params = {"W1": torch.randn(d, ffn, generator=gen, device=DEV) * d ** -0.5, "b1": torch.zeros(ffn, device=DEV),
                       "W2": torch.randn(ffn, d, generator=gen, device=DEV) * ffn ** -0.5, "b2": torch.zeros(d, device=DEV)}
        self.copies = {k: v.to(torch.bfloat16) for k, v in self.params.items()}
        self.z, self.a, self.out, self.dz = _bf16(tokens, ffn), _bf16(tokens, ffn), _bf16(tokens, d), _bf16(tokens, ffn)
        self.second = PlannedGemms([(tokens, ffn, d, 0, 1), (ffn, d, tokens, 1, 0)], devices)     # dout W2^T, a^T dout
        self.first = PlannedGemms([(tokens, d, ffn, 0, 1), (d, ffn, tokens, 1, 0)], devices)      # dz W1^T, y^T dz
        self.grads = {"W1": self.first.C[1], "b1": torch.empty(ffn, device=DEV), "W2": self.second.C[1], "b2": torch.empty(d, device=DEV)}

    def forward(self, x, residual):
        w, (y, h) = self.copies, self.norm.forward(x, residual)
        cl.linear(y, w["W1"], self.a, bias=self.params["b1"], act="gelu_tanh", z=self.z)
        cl.linear(self.a, w["W2"], self.out, bias=self.params["b2"])
        return self.out, h

    def backward(self, dh):
        """dh: gradient of h + out.  Returns the gradient of h."""
        w, dout = self.copies, dh.to(torch.bfloat16)
        da, _ = self.second.run([dout, self.a], [w["W2"], dout])
        cl.act_backward(dout, None, dbias=self.grads["b2"])
        cl.act_backward(da, self.z, self.dz, act="gelu_tanh", dbias=self.grads["b1"])
        dy, _ = self.first.run([self.dz, self.norm.y], [w["W1"], self.dz])
        return self.norm.backward(dy, dh)


class Model:
    """`step` leaves the loss of each token and the gradients of all parameters."""

    def __init__(self, tokens=1024, vocab=2000, d=256, ffn=768, blocks=2, n_devices=24, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        devices = ci.make_devices(n_devices, 64 * ci.MB, ci.GB, seed)
        self.tokens, self.vocab, self.d = tokens, vocab, d
        self.scale = d ** 0.5
        self.table = torch.randn(vocab, d, generator=gen, device=DEV) * d ** -0.5
        self.table_copy = self.table.to(torch.bfloat16)
        self.blocks = [Block(tokens, d, ffn, devices, gen) for _ in range(blocks)]
        self.last = Norm(tokens, d)
        self.x = _bf16(tokens, d)
        self.none = torch.zeros(tokens, d, device=DEV)
        self.scores, self.dscores = _bf16(tokens, vocab), _bf16(tokens, vocab)
        self.logp, self.lse, self.loss = (torch.empty(tokens, device=DEV) for _ in range(3))
        self.head = PlannedGemms([(tokens, d, vocab, 0, 0), (vocab, d, tokens, 1, 0)], devices)    # dscores E, dscores^T y
        self.table_grad = self.head.C[1]
        self.params, self.grads, self.copies, self.decay = {"table": self.table}, {"table": self.table_grad}, {"table": self.table_copy}, {"table": 0.0}
        for i, b in enumerate(self.blocks + [self.last]):
            for name, part in (("norm.", b.norm), ("", b)) if isinstance(b, Block) else (("norm.", b),):
                for k in part.params:
                    at = f"{i}.{name}{k}"
                    self.params[at], self.grads[at] = part.params[k], part.grads[k]
                    self.copies[at] = part.copies[k] if hasattr(part, "copies") else None
                    self.decay[at] = 0.01 if k in ("W1", "W2") else 0.0

    def step(self, tokens, targets, teacher=None):
        """teacher: (index, values) of its best scores, [tokens, k]; without one, the targets' cross entropy (PADDING: not counted)."""
        cl.embedding(tokens, self.table_copy, self.x, scale=self.scale)
        out, h = self.x, self.none
        for b in self.blocks:
            out, h = b.forward(out, h)
        y, _ = self.last.forward(out, h)
        cl.linear(y, self.table_copy, self.scores, transB=True)
        share = torch.full((self.tokens,), 1.0 / self.tokens, device=DEV)
        if teacher is None:
            cl.token_logprobs(self.scores, targets, self.logp, lse=self.lse)
            cl.token_logprobs_backward(self.scores, targets, self.lse, self.dscores, dlogp=-share)
            torch.neg(self.logp, out=self.loss)
        else:
            cl.distill(self.scores, *teacher, self.loss, lse=self.lse)
            cl.distill_backward(self.scores, *teacher, self.lse, share, self.dscores)
        dy, _ = self.head.run([self.dscores, self.dscores], [self.table_copy, y])
        dh = self.last.backward(dy, None)
        for b in reversed(self.blocks):
            dh = b.backward(dh)
        cl.embedding_backward(dh, tokens, self.table_grad, scale=self.scale, accumulate=True)
        return self.loss

    def check(self):
        assert cl.linear_status() == 0
        for p in [self.head] + [g for b in self.blocks for g in (b.first, b.second)]:
            p.plan.check_status()


def batch(model, step, seed=0):
    """Tokens whose frequency falls with their rank, each one's next token by a fixed map, and a tenth of padding at the end."""
    gen = torch.Generator(device=DEV).manual_seed(1000003 * seed + step)
    u = torch.rand(model.tokens, generator=gen, device=DEV)
    tokens = (model.vocab ** u - 1).long().clamp_(0, model.vocab - 1)
    targets = (tokens * 7 + 3) % model.vocab
    targets[model.tokens - model.tokens // 10:] = PADDING
    return tokens, targets


def teacher_of(targets, vocab, k=8):
    """A teacher that is sure of the next token but for a few others: its k best scores; padded rows are empty."""
    at = (targets[:, None] + 11 * torch.arange(k, device=DEV)) % vocab
    at[targets < 0] = -1
    values = 4.0 - 1.5 * torch.arange(k, device=DEV, dtype=torch.float32).expand(len(targets), k)
    return at.to(torch.int32), values.contiguous()


def optimizer(model):
    """AdamW over all of the model's parameters, in their order."""
    names = list(model.params)
    params = [model.params[k].view(-1) for k in names]
    copies = [None if model.copies[k] is None else model.copies[k].view(-1) for k in names]
    return cl.AdamW(params, [model.grads[k].view(-1) for k in names], [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params],
                    copies=copies, weight_decay=[model.decay[k] for k in names])


def train(steps=60, teacher=False, lr=2e-3, seed=0, **size):
    """Mean losses of `steps` steps."""
    model = Model(seed=seed, **size)
    opt, losses = optimizer(model), []
    for step in range(1, steps + 1):
        tokens, targets = batch(model, step, seed)
        losses.append(model.step(tokens, targets, teacher_of(targets, model.vocab) if teacher else None).mean())
        opt.step(step=step, lr=lr)
    model.check()
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--teacher", action="store_true")
    args = ap.parse_args()
    for i, v in enumerate(train(args.steps, args.teacher)):
        if i % 10 == 0 or i == args.steps - 1:
            print(f"step {i + 1:4d}  loss {v:.5f}")
