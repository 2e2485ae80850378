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


@pytest.mark.parametrize("with_teacher", [False, True])
def test_updates_reach_the_next_step(with_teacher):
    """The weights after each step are AdamW's of the step's own gradients, to the bit, in the copies that the products read too; the
    second step's loss and gradients are those of the updated weights (tolerances as in test_a_steps_loss_and_gradients)."""
    from oracle import ops as ref
    from train_token_model import Model, batch, optimizer, teacher_of
    model = Model(seed=6, **SIZE)
    opt, lr = optimizer(model), 2e-3
    flat = lambda t: t.detach().float().cpu().numpy().ravel()  # noqa: E731
    state = {k: (0 * flat(p), 0 * flat(p)) for k, p in model.params.items()}
    for step in (1, 2):
        tokens, targets = batch(model, step, 6)
        teacher = teacher_of(targets, model.vocab) if with_teacher else None
        want, grads = _torch_step(model, tokens, targets, teacher)
        got = model.step(tokens, targets, teacher)
        assert float((got - want).abs().max()) < 0.15
        for k, g in model.grads.items():
            off = float((g - grads[k]).norm() / grads[k].norm())
            assert off < 0.03, f"step {step}, {k}: {off:.4f}"
        before = {k: (flat(p), flat(model.grads[k])) for k, p in model.params.items()}
        opt.step(step=step, lr=lr)
        torch.cuda.synchronize()
        for k, p in model.params.items():
            new, m, v = ref.adamw(*before[k], *state[k], lr=lr, beta1=0.9, beta2=0.999, eps=1e-8, step=step, weight_decay=model.decay[k])
            state[k] = m, v
            assert (flat(p) == new).all() and (new != before[k][0]).any(), f"step {step}, {k}"
            if model.copies[k] is not None:
                assert torch.equal(model.copies[k], p.to(torch.bfloat16)), f"step {step}, {k}"
    model.check()
