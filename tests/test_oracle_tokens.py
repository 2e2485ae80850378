"""The oracle of the operators on tokens, pinned: against torch's own functions in 64 bits, and the gradients against
central differences of the forward passes."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as ref


def _rng(seed):
    return np.random.default_rng(seed)


def _difference(f, x, h=1e-5):
    """Central differences of the scalar f at every element of x."""
    g = np.zeros(x.shape)
    for at in np.ndindex(*x.shape):
        hi, lo = x.copy(), x.copy()
        hi[at] += h
        lo[at] -= h
        g[at] = (f(hi) - f(lo)) / (2 * h)
    return g


def test_embedding_and_its_gradient():
    rng = _rng(1)
    table, tokens = rng.normal(size=(9, 5)), np.array([3, 0, 8, 3, -1, 9, 2 ** 40, 3, -100])
    got = ref.embedding(tokens, table, 2.0)
    assert np.array_equal(got[[0, 1, 2]], 2 * table[[3, 0, 8]]) and not got[[4, 5, 6, 8]].any()
    dy = rng.normal(size=got.shape)
    want = _difference(lambda t: float((ref.embedding(tokens, t, 2.0) * dy).sum()), table)
    grad, _, count = ref.embedding_backward(dy, tokens, 9, 2.0)
    assert np.allclose(grad, want, atol=1e-8) and count.tolist() == [1, 0, 0, 3, 0, 0, 0, 0, 1]
    assert np.allclose(ref.embedding_backward(dy, tokens, 9, 2.0, table)[0], want + table, atol=1e-8)


def test_layernorm_and_its_gradient():
    rng = _rng(2)
    x, r, w, b = rng.normal(size=(4, 7)), rng.normal(size=(4, 7)), rng.normal(size=7), rng.normal(size=7)
    h, y, mean, rstd = ref.layernorm(x, r, w, b, 1e-3)
    t = torch.nn.functional.layer_norm(torch.tensor(x + r), (7,), torch.tensor(w), torch.tensor(b), 1e-3)
    assert np.allclose(y, t.numpy(), atol=1e-13) and np.array_equal(h, x + r)
    dy, dres = rng.normal(size=y.shape), rng.normal(size=y.shape)
    dx, dw, db = ref.layernorm_backward(dy, h, w, mean, rstd, dres)
    f = lambda x, w, b: float((ref.layernorm(x, r, w, b, 1e-3)[1] * dy).sum())  # noqa: E731
    assert np.allclose(dx, _difference(lambda v: f(v, w, b), x) + dres, atol=1e-8)
    assert np.allclose(dw, _difference(lambda v: f(x, v, b), w), atol=1e-8) and np.allclose(db, _difference(lambda v: f(x, w, v), b), atol=1e-8)


@pytest.mark.parametrize("scale", [1.0, 0.5, 2.0])
def test_logprobs_and_their_gradient(scale):
    rng = _rng(3)
    x, tokens = rng.normal(size=(5, 11)) * 3, np.array([4, 0, 10, -100, 11])
    logp, lse, entropy, values, index = ref.logprobs(x, tokens, scale, 4)
    t = torch.log_softmax(torch.tensor(x) * scale, 1)
    assert np.allclose(logp[:3], t[range(3), tokens[:3]].numpy()) and not logp[3:].any()
    assert np.allclose(lse, torch.logsumexp(torch.tensor(x) * scale, 1).numpy())
    assert np.allclose(entropy, torch.distributions.Categorical(logits=torch.tensor(x) * scale).entropy().numpy())
    best = t.topk(4)
    assert np.allclose(values, best.values.numpy()) and np.array_equal(index, best.indices.numpy())
    up, z, e = rng.normal(size=5), rng.normal(size=5), rng.normal(size=5)

    def f(v):
        a, b, c, _, _ = ref.logprobs(v, tokens, scale)
        return float((a * up + b * z + c * e).sum())
    dx, _ = ref.logprobs_backward(x, tokens, lse, scale, up, z, e, entropy)
    assert np.allclose(dx, _difference(f, x), atol=1e-7)


def test_logprobs_of_masked_and_broken_rows():
    inf, low = np.inf, float(np.finfo(np.float32).min)
    x = np.array([[-inf, -inf, -inf], [low, low, -inf], [1.0, -inf, low], [np.nan, 0, 1], [inf, 0, 1], [0.0, -0.0, 0.0]])
    logp, lse, entropy, values, index = ref.logprobs(x, np.array([1, 0, 0, 1, 1, 2]), 1.0, 3)
    assert logp[0] == logp[1] == -inf and lse[0] == lse[1] == -inf and entropy[0] == entropy[1] == 0 and (values[:2] == -inf).all()
    assert logp[2] == 0 and lse[2] == 1 and entropy[2] == 0 and index.tolist() == [[0, 1, 2], [0, 1, 2], [0, 2, 1], [0, 2, 1], [0, 2, 1], [0, 1, 2]]
    assert np.isnan(logp[3:5]).all() and np.isnan(lse[3:5]).all() and np.isnan(entropy[3:5]).all() and np.isnan(values[3:5]).all()
    dx, _ = ref.logprobs_backward(x[:3], np.array([1, 0, 0]), lse[:3], 1.0, np.ones(3), np.ones(3), np.ones(3), entropy[:3])
    assert not dx[:2].any() and np.allclose(dx[2], [1.0, 0, 0])


@pytest.mark.parametrize("normalize", [False, True])
def test_distill_and_its_gradient(normalize):
    rng = _rng(4)
    x = rng.normal(size=(4, 9))
    index = np.array([[1, 5, 1, 8], [0, -1, 9, 3], [-1, -1, -1, -1], [2, 2, 2, 2]])
    values = rng.normal(size=(4, 4)) - 2
    values[3, 1] = -np.inf
    loss, lse, _ = ref.distill(x, index, values, 0.5, normalize)
    dloss = rng.normal(size=4)
    dx, _ = ref.distill_backward(x, index, values, lse, dloss, 0.5, normalize)
    want = _difference(lambda v: float((ref.distill(v, index, values, 0.5, normalize)[0] * dloss).sum()), x)
    assert np.allclose(dx, want, atol=1e-8) and loss[2] == 0 and not dx[2].any()
    # a teacher that names every place once: the divergence of two distributions
    full = np.arange(9)[None].repeat(4, 0)
    t = rng.normal(size=(4, 9))
    if normalize:
        p, q = torch.log_softmax(torch.tensor(x) * 0.5, 1), torch.log_softmax(torch.tensor(t) * 0.5, 1)
        assert np.allclose(ref.distill(x, full, t, 0.5)[0], torch.nn.functional.kl_div(p, q, log_target=True, reduction="none").sum(1).numpy())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("normalize", [True, False])
def test_a_broken_teacher_leaves_its_empty_entries_empty(bad, normalize):
    index, values = np.array([3, 5, -1, 9, 2]), np.array([0.5, bad, bad, 0.1, -1.0])
    q, log_q = ref.teacher(index, values, 9, 1.3, normalize)
    live = [0, 1, 4]
    with np.errstate(invalid="ignore"):
        want = torch.softmax(torch.tensor(1.3 * values[live]), 0) if normalize else torch.exp(torch.tensor(1.3 * values[live]))
    assert not q[[2, 3]].any() and np.all(log_q[[2, 3]] == -math.inf)
    np.testing.assert_allclose(q[live], want.numpy(), rtol=1e-12)
    x = np.linspace(-1, 1, 18).reshape(2, 9)
    loss, _, _ = ref.distill(x, np.stack([index, [-1, -1, -1, -1, 10]]), np.stack([values, np.full(5, bad)]), 1.3, normalize)
    assert not math.isfinite(loss[0]) and loss[1] == 0
