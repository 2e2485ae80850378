"""CPU oracle of the operators around the GEMMs: AdamW with 32- and 8-bit states, root-mean-square norm and its
backward pass, rows in 8 bits, the product with an epilogue and that epilogue's backward pass.

NumPy and SciPy's erfc only; test infrastructure.  Everything is computed in fp64 from the definitions, except `adamw`, whose
definition says how each operation is rounded to fp32: there the stored bits themselves are the result.
"""
from __future__ import annotations

import math

import numpy as np
from scipy import special

M64 = (1 << 64) - 1
BLOCK = 256
E4M3_MAX = 448.0


# ---- E4M3 ---------------------------------------------------------------------------------------------
def e4m3_table() -> np.ndarray:
    """Value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    out = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        if c & 0x7F == 0x7F:
            v = math.nan
        out[c] = -v if c & 0x80 else v
    return out


def e4m3_step(q):
    """Distance of neighbouring codes around magnitudes q (fp64)."""
    a = np.maximum(np.abs(np.asarray(q, dtype=np.float64)), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(a)) - 3)


# ---- AdamW ----------------------------------------------------------------------------------------------
def mix64(x: np.ndarray) -> np.ndarray:
    """SplitMix64's output function."""
    with np.errstate(over="ignore"):
        x = np.asarray(x, dtype=np.uint64) + np.uint64(0x9E3779B97F4A7C15)
        x = (x ^ (x >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        x = (x ^ (x >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return x ^ (x >> np.uint64(31))


def random_bits(seed: int, step: int, tensor: int, n: int):
    """The 16 random bits of each element for m and for v."""
    base = np.array([(seed + (step << 32) + tensor) & M64], dtype=np.uint64)
    key = mix64(mix64(base))[0]
    e = np.arange(n, dtype=np.uint64)
    with np.errstate(over="ignore"):
        word = mix64(key + (e >> np.uint64(1)))
    word = word >> ((e & np.uint64(1)) * np.uint64(32))
    return (word & np.uint64(0xFFFF)).astype(np.int64), ((word >> np.uint64(16)) & np.uint64(0xFFFF)).astype(np.int64)


def stochastic_codes(q: np.ndarray, u: np.ndarray) -> np.ndarray:
    """Magnitude codes of fp32 values |q| <= 448 from their bracketing codes: up when fraction + u / 2^16 >= 1."""
    out = np.empty(q.shape, dtype=np.uint8)
    table = e4m3_table()[:0x7F]
    for i, (x, r) in enumerate(zip(np.abs(q).astype(np.float64), u)):
        if math.isnan(x):
            out[i] = 0x7F
            continue
        lo = int(np.searchsorted(table, x, side="right")) - 1
        if lo >= 0x7E:
            out[i] = 0x7E
            continue
        if x >= 2.0 ** -6:            # 20 bits are cut: the random bits stand on top of them
            cut = (x - table[lo]) / (table[lo + 1] - table[lo]) * 2 ** 20
            up = cut + int(r) * 16 >= 2 ** 20
        else:                         # the sum is rounded to fp32
            up = math.floor(np.float32(np.float32(x) * np.float32(512)) + np.float32(int(r) / 65536)) > lo
        out[i] = lo + 1 if up else lo
    return out


def _scale(top: np.float32):
    if top < np.float32(2.0 ** -100):
        return np.float32(0), np.float32(0)
    s = np.float32(top * np.float32(1 / E4M3_MAX))
    return s, np.float32(np.float32(1) / s)


def adamw(p, g, m, v, *, lr, beta1, beta2, eps, step, weight_decay, grad_scale=1.0, m_scale=None, v_scale=None, seed=0, tensor=0):
    """One step on flat arrays, every operation rounded to fp32.  32-bit states: (p, m, v) fp32.  8-bit states
    (m, v: uint8 codes with m_scale, v_scale): (p, m codes, v codes, m_scale, v_scale)."""
    f = np.float32
    with np.errstate(all="ignore"):
        p, g = p.astype(f), g.astype(f) * f(grad_scale)
        n = len(p)
        eight = m_scale is not None
        if eight:
            table = e4m3_table().astype(f)
            block = np.arange(n) // BLOCK
            mo = table[m] * m_scale[block]
            root = table[v] * v_scale[block]
            vo = root * root
        else:
            mo, vo = m.astype(f), v.astype(f)
        mo = mo * f(beta1) + g * f(1.0 - beta1)
        vo = vo * f(beta2) + (g * g) * f(1.0 - beta2)
        r = np.sqrt(vo)
        den = r * f(1.0 / math.sqrt(1.0 - math.pow(beta2, step))) + f(eps)
        p = p * f(1.0 - lr * weight_decay) - (mo / den) * f(lr / (1.0 - math.pow(beta1, step)))
        if not eight:
            return p, mo, vo
        um, uv = random_bits(seed, step, tensor, n)
        cm, cv = np.zeros(n, dtype=np.uint8), np.zeros(n, dtype=np.uint8)
        sm, sv = np.zeros(-(-n // BLOCK), dtype=f), np.zeros(-(-n // BLOCK), dtype=f)
        for b in range(len(sm)):
            at = slice(b * BLOCK, min(n, (b + 1) * BLOCK))
            sm[b], im = _scale(np.max(np.abs(mo[at])))
            sv[b], iv = _scale(np.max(r[at]))
            qm, qv = mo[at] * im, r[at] * iv
            cm[at] = stochastic_codes(qm, um[at]) | np.where(qm < 0, 0x80, 0).astype(np.uint8)
            c = stochastic_codes(qv, uv[at])
            cv[at] = np.where((c == 0) & (qv > 0), 1, c)
        return p, cm, cv, sm, sv


# ---- norm -------------------------------------------------------------------------------------------------
def rmsnorm(x, r, w, eps):
    """(h, y, rstd) in fp64."""
    h = x if r is None else x + r
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    y = h * rstd[:, None]
    return h, (y if w is None else y * w), rstd


def rmsnorm_backward(dy, h, w, rstd, dres=None):
    """(dx, dw) in fp64."""
    xh = h * rstd[:, None]
    q = dy if w is None else dy * w
    dx = rstd[:, None] * (q - xh * np.mean(q * xh, axis=1, keepdims=True))
    return (dx if dres is None else dx + dres), np.sum(dy * xh, axis=0)


# ---- product with an epilogue --------------------------------------------------------------------------------
def _phi(z):
    return 0.5 * special.erfc(-z / math.sqrt(2.0))


def act(z, kind):
    if kind == "relu":
        return np.maximum(z, 0.0)
    if kind == "gelu":
        return z * _phi(z)
    if kind == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if kind == "silu":
        return z / (1.0 + np.exp(-z))
    return z


def act_slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "gelu":
        return _phi(z) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def linear(A, B, *, scale_a=None, scale_b=None, bias=None, kind="none", mul=None, res=None):
    """(C, z) in fp64; A [M, K] and B [K, N] as the product sees them."""
    z = A @ B
    if scale_a is not None:
        z = z * scale_a[:, None]
    if scale_b is not None:
        z = z * scale_b
    if bias is not None:
        z = z + bias
    c = act(z, kind)
    if mul is not None:
        c = c * mul
    if res is not None:
        c = c + res
    return c, z


def act_backward(dy, z, kind, mul=None):
    """(dz, dmul, dbias) in fp64."""
    one = np.ones_like(dy) if kind == "none" else act_slope(z, kind)
    dz = dy * one if mul is None else dy * one * mul
    return dz, (None if z is None else dy * act(z, kind)), dz.sum(axis=0)
