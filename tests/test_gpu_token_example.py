"""The operators on tokens together with planned GEMMs: the example's step against the same model written with torch in fp32, loss and
gradients, and that its training runs."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
SIZE = dict(tokens=512, vocab=1000, d=128, ffn=384, blocks=2, n_devices=12)


def _torch_step(model, tokens, targets, teacher):
    """Loss of each token and gradients of the mean, with fp32 arithmetic from the bf16 weights that the products read."""
    p = {k: (model.copies[k].float() if model.copies[k] is not None and model.params[k].dim() == 2 else model.params[k].clone()).requires_grad_() for k in model.params}
    norm = lambda h, at: torch.nn.functional.layer_norm(h, (model.d,), p[at + "w"], p[at + "b"], 1e-5)  # noqa: E731
    h = p["table"][tokens] * model.scale
    for i in range(len(model.blocks)):
        y = norm(h, f"{i}.norm.")
        h = h + torch.nn.functional.gelu(y @ p[f"{i}.W1"] + p[f"{i}.b1"], approximate="tanh") @ p[f"{i}.W2"] + p[f"{i}.b2"]
    logp = torch.log_softmax(norm(h, f"{len(model.blocks)}.norm.") @ p["table"].t(), 1)
    if teacher is None:
        loss = torch.where(targets >= 0, -logp.gather(1, targets.clamp_min(0)[:, None])[:, 0], 0.0)
    else:
        index, values = teacher
        live = (index >= 0)[:, :1]
        q = torch.softmax(values, 1)
        loss = torch.where(live, q * (torch.log(q) - logp.gather(1, index.long().clamp_min(0))), 0.0).sum(1)
    loss.mean().backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("with_teacher", [False, True])
def test_a_steps_loss_and_gradients(with_teacher):
    from train_token_model import Model, batch, teacher_of
    model = Model(seed=5, **SIZE)
    tokens, targets = batch(model, 1, 5)
    teacher = teacher_of(targets, model.vocab) if with_teacher else None
    want, grads = _torch_step(model, tokens, targets, teacher)
    got = model.step(tokens, targets, teacher)
    model.check()
    # bf16 between the operators: a rounding is off by 2^-9 of a value on average (2^-8 at most).  Scores of size 10 are rounded once: 0.04
    # at most, and their operands' roundings average out over 128 terms; a loss is a difference of two of them.
    assert float((got - want).abs().max()) < 0.15
    assert not got[targets < 0].any()
    # A gradient passes up to four roundings on its way through each of two blocks and three more at the ends: eleven of 2^-9 each,
    # independent of each other: 0.0065 of its norm, and as much again from the rounded activations that it is multiplied with.
    for k, g in model.grads.items():
        off = float((g - grads[k]).norm() / grads[k].norm())
        assert off < 0.03, f"{k}: {off:.4f}"


@pytest.mark.parametrize("with_teacher", [False, True])
def test_training_runs(with_teacher):
    from train_token_model import train
    losses = train(steps=6, teacher=with_teacher, seed=1, **SIZE)
    assert len(losses) == 6 and all(v == v and abs(v) < 1e3 for v in losses)
