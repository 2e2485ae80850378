"""Pins of the operators' oracle: E4M3 against torch's type, stochastic rounding against its expectation and its
brackets, AdamW against the textbook recursion, every gradient against central differences."""
import math

import numpy as np
import pytest
import torch

from oracle import ops

KINDS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def test_e4m3_values_are_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(ops.e4m3_table(), want, equal_nan=True)
    assert ops.e4m3_table()[0x7E] == 448.0 and ops.e4m3_table()[1] == 2.0 ** -9


def test_mix64_is_splitmix64():
    # the generator's first outputs for state 1234567: state advances by the golden gamma before each output
    state, outs = 1234567, []
    for _ in range(3):
        outs.append(int(ops.mix64(np.uint64(state))))
        state = (state + 0x9E3779B97F4A7C15) & ops.M64
    assert outs == [6457827717110365317, 3203168211198807973, 9817491932198370423]


def test_stochastic_codes_bracket_and_average():
    rng = np.random.default_rng(0)
    q = np.concatenate([rng.uniform(0, 0.03, 300), 448 * rng.uniform(0, 1, 300) ** 4, [0.0, 448.0, 2 ** -9, 2 ** -6, 447.9]]).astype(np.float32)
    table = ops.e4m3_table()
    low, high = ops.stochastic_codes(q, np.zeros(len(q), dtype=np.int64)), ops.stochastic_codes(q, np.full(len(q), 65535))
    assert np.all(table[low] <= q) and np.all(table[high] >= q - 2.0 ** -15 * ops.e4m3_step(q))
    assert np.all(high.astype(int) - low <= 1)
    exact = table[low] == q                                    # a value that is a code stays one
    assert exact.sum() >= 4 and np.array_equal(low[exact], high[exact])
    # the mean over all random bits is the value itself (16 bits: up to 2^-16 of a step)
    for x in (0.0033, 0.4, 3.3, 100.0, 440.0):
        u = np.arange(0, 65536, 16)
        mean = table[ops.stochastic_codes(np.full(len(u), x, dtype=np.float32), u)].mean()
        assert abs(mean - x) <= 2.0 ** -11 * float(ops.e4m3_step(x))


def test_adamw_is_the_textbook_recursion():
    rng = np.random.default_rng(1)
    n, lr, b1, b2, eps, wd = 64, 1e-2, 0.9, 0.99, 1e-8, 0.1
    p = rng.normal(size=n)
    p32, m32, v32 = p.astype(np.float32), np.zeros(n, np.float32), np.zeros(n, np.float32)
    p64, m64, v64 = p32.astype(np.float64), np.zeros(n), np.zeros(n)
    for t in range(1, 6):
        g = rng.normal(size=n).astype(np.float32)
        p32, m32, v32 = ops.adamw(p32, g, m32, v32, lr=lr, beta1=b1, beta2=b2, eps=eps, step=t, weight_decay=wd)
        m64 = b1 * m64 + (1 - b1) * g.astype(np.float64)
        v64 = b2 * v64 + (1 - b2) * g.astype(np.float64) ** 2
        p64 = p64 - lr * wd * p64 - lr * (m64 / (1 - b1 ** t)) / (np.sqrt(v64 / (1 - b2 ** t)) + eps)
    # five steps of about ten roundings each, each at most 2^-24 of values of the size of p or of lr
    assert np.allclose(p32, p64, rtol=0, atol=60 * 2.0 ** -24 * np.abs(p64).max())
    # torch's optimizer, in 64 bits
    q = torch.tensor(p, dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([q], lr=lr, betas=(b1, b2), eps=eps, weight_decay=wd)
    rng = np.random.default_rng(1)
    rng.normal(size=n)
    for _ in range(5):
        q.grad = torch.tensor(rng.normal(size=n).astype(np.float32).astype(np.float64))
        opt.step()
    assert np.allclose(p32, q.detach().numpy(), rtol=0, atol=60 * 2.0 ** -24 * np.abs(p64).max())


def _differences(f, x, direction, h=1e-5):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


@pytest.mark.parametrize("weight", [True, False])
def test_norm_gradient_against_differences(weight):
    rng = np.random.default_rng(2)
    x, r, w = rng.normal(size=(5, 24)), rng.normal(size=(5, 24)), (rng.normal(size=24) if weight else None)
    dy, dres = rng.normal(size=(5, 24)), rng.normal(size=(5, 24))

    def loss(x_, w_):
        h, y, _ = ops.rmsnorm(x_, r, w_, 1e-3)
        return np.sum(dy * y) + np.sum(dres * h)
    h, _, rstd = ops.rmsnorm(x, r, w, 1e-3)
    dx, dw = ops.rmsnorm_backward(dy, h, w, rstd, dres)
    for _ in range(4):
        d = rng.normal(size=x.shape)
        assert np.isclose(np.sum(dx * d), _differences(lambda t: loss(t, w), x, d), rtol=1e-6, atol=1e-8)
        if weight:
            e = rng.normal(size=24)
            assert np.isclose(np.sum(dw * e), _differences(lambda t: loss(x, t), w, e), rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gated", [False, True])
def test_epilogue_gradient_against_differences(kind, gated):
    rng = np.random.default_rng(3)
    A, B, bias = rng.normal(size=(6, 9)), rng.normal(size=(9, 7)), rng.normal(size=7)
    mul = rng.normal(size=(6, 7)) if gated else None
    dy = rng.normal(size=(6, 7))
    _, z = ops.linear(A, B, bias=bias, kind=kind, mul=mul)
    dz, dmul, db = ops.act_backward(dy, z, kind, mul)
    dA, dB = dz @ B.T, A.T @ dz

    def loss(a, b, c, u):
        return np.sum(dy * ops.linear(a, b, bias=c, kind=kind, mul=u)[0])
    for base, grad, f in ((A, dA, lambda t: loss(t, B, bias, mul)), (B, dB, lambda t: loss(A, t, bias, mul)),
                          (bias, db, lambda t: loss(A, B, t, mul))):
        d = rng.normal(size=base.shape)
        assert np.isclose(np.sum(grad * d), _differences(f, base, d), rtol=1e-5, atol=1e-7)
    if gated:
        d = rng.normal(size=mul.shape)
        assert np.isclose(np.sum(dmul * d), _differences(lambda t: loss(A, B, bias, t), mul, d), rtol=1e-6, atol=1e-8)


def test_activations_are_torchs():
    z = torch.linspace(-8, 8, 401, dtype=torch.float64)
    want = {"relu": torch.relu(z), "gelu": torch.nn.functional.gelu(z), "gelu_tanh": torch.nn.functional.gelu(z, approximate="tanh"),
            "silu": torch.nn.functional.silu(z), "none": z}
    for kind in KINDS:
        assert np.allclose(ops.act(z.numpy(), kind), want[kind].numpy(), rtol=1e-12, atol=1e-14), kind
    assert math.isclose(ops.act(np.array([1.0]), "gelu")[0], 0.8413447460685429)
