"""The operators around the GEMMs on the GPU against their 64-bit oracle (AdamW: against its exact fp32 definition,
bit for bit).  Tolerances are the roundings of the stated arithmetic: U = 2^-24 is half a unit of fp32, a bf16
result may be half a unit of its 8 significant bits (2^-8) off, sums of n terms in fp32 a modest multiple of sqrt(n) U of their
terms' magnitudes (bounded here by a fixed 64 U, well above any order of up to 2^15 terms split over lanes)."""
import numpy as np
import pytest
import torch

from oracle import ops as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SUM = 64 * U
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
KINDS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def cl():
    import paper_2512_22142_b200 as cl
    return cl


def _dev():
    return torch.device("cuda:0")


def _rand(rng, shape, dtype, scale=1.0):
    return torch.tensor(rng.normal(size=shape) * scale, dtype=torch.float32).to(dtype).to(_dev())


def _f64(t):
    return None if t is None else t.to(torch.float64).cpu().numpy()


def _close(got, want, abs_tol, what=""):
    """|got - want| <= abs_tol + the rounding of got's type."""
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    g = _f64(got)
    assert np.isfinite(g).all(), what
    bad = np.abs(g - want) - (abs_tol + half * np.maximum(np.abs(want), np.abs(g)) * 1.001 + 1e-38)
    assert bad.max(initial=-1.0) <= 0, f"{what}: {bad.max():.3e} over at {np.unravel_index(np.argmax(bad), bad.shape)}"


def _strided(rng, rows, cols, dtype, pad, scale=1.0):
    """A [rows, cols] view whose rows lie `cols + pad` apart."""
    return _rand(rng, (max(rows, 1), cols + pad), dtype, scale)[:rows, :cols]


# ---- AdamW ---------------------------------------------------------------------------------------------
def _adam_state(rng, sizes, eight, grad, copies, shift=0):
    """Tensors whose storage begins `shift` elements into an allocation (shift != 0: the narrow path)."""
    out = dict(p=[], g=[], m=[], v=[], ms=[], vs=[], w=[])
    for n in sizes:
        cut = lambda t: t.to(_dev())[shift:]  # noqa: E731
        N = n + shift
        out["p"].append(cut(torch.tensor(rng.normal(size=N) * 0.02, dtype=torch.float32)))
        out["g"].append(cut(torch.tensor(rng.normal(size=N) * 0.01, dtype=torch.float32).to(grad)))
        m, v = rng.normal(size=N) * 0.003, (rng.normal(size=N) * 0.01) ** 2
        if eight:
            codes = torch.tensor(rng.integers(0, 0x7F, size=N), dtype=torch.uint8)
            sign = torch.tensor(rng.integers(0, 2, size=N) * 0x80, dtype=torch.uint8)
            out["m"].append(cut(codes | sign).view(torch.float8_e4m3fn))
            out["v"].append(cut(torch.tensor(rng.integers(0, 0x7F, size=N), dtype=torch.uint8)).view(torch.float8_e4m3fn))
            blocks = -(-n // 256)
            out["ms"].append(torch.tensor(rng.uniform(1e-6, 1e-5, size=blocks), dtype=torch.float32).to(_dev()))
            out["vs"].append(torch.tensor(rng.uniform(1e-6, 1e-4, size=blocks), dtype=torch.float32).to(_dev()))
        else:
            out["m"].append(cut(torch.tensor(m, dtype=torch.float32)))
            out["v"].append(cut(torch.tensor(v, dtype=torch.float32)))
        if copies:
            out["w"].append(cut(torch.zeros(N, dtype=torch.bfloat16)))
    return out


def _make(cl, s, wd, eight, copies):
    return cl.AdamW(s["p"], s["g"], s["m"], s["v"], copies=s["w"] if copies else None, m_scales=s["ms"] if eight else None,
                    v_scales=s["vs"] if eight else None, weight_decay=wd)


def _codes(t):
    return t.view(torch.uint8).cpu().numpy()


def _bits(t):
    return t.cpu().view(torch.int32).numpy()


def _check_step(s0, s, wd, eight, copies, hyper, step, seed):
    for i in range(len(s["p"])):
        if s["p"][i].numel() == 0:
            continue
        args = dict(lr=hyper["lr"], beta1=hyper["beta1"], beta2=hyper["beta2"], eps=hyper["eps"], step=step, weight_decay=wd[i],
                    grad_scale=hyper.get("grad_scale", 1.0), seed=seed, tensor=i)
        p, g = s0["p"][i].cpu().numpy(), s0["g"][i].float().cpu().numpy()
        if eight:
            want = ref.adamw(p, g, _codes(s0["m"][i]), _codes(s0["v"][i]), m_scale=s0["ms"][i].cpu().numpy(), v_scale=s0["vs"][i].cpu().numpy(), **args)
            assert np.array_equal(_codes(s["m"][i]), want[1]), f"tensor {i}: codes of m"
            assert np.array_equal(_codes(s["v"][i]), want[2]), f"tensor {i}: codes of v"
            assert np.array_equal(_bits(s["ms"][i]), want[3].view(np.int32)) and np.array_equal(_bits(s["vs"][i]), want[4].view(np.int32))
        else:
            want = ref.adamw(p, g, s0["m"][i].cpu().numpy(), s0["v"][i].cpu().numpy(), **args)
            assert np.array_equal(_bits(s["m"][i]), want[1].view(np.int32)) and np.array_equal(_bits(s["v"][i]), want[2].view(np.int32))
        assert np.array_equal(_bits(s["p"][i]), want[0].astype(np.float32).view(np.int32)), f"tensor {i}: weights"
        if copies:
            assert torch.equal(s["w"][i].cpu(), torch.tensor(want[0]).to(torch.bfloat16))


def _clone(s):
    return {k: [t.clone() for t in v] for k, v in s.items()}


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw_stored_bits_are_the_definitions(cl, eight, grad, shift):
    rng = np.random.default_rng(10)
    sizes = [1, 0, 255, 256, 257, 2048, 5000, 3, 2049]
    wd = [0.1, 0.0, 0.3, 0.0, 0.1, 0.01, 0.0, 1.0, 0.1]
    copies = grad == "bf16"
    s = _adam_state(rng, sizes, eight, DT[grad], copies, shift)
    opt = _make(cl, s, wd, eight, copies)
    hyper = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-6, grad_scale=0.5)
    for step in (1, 2, 1000):
        before = _clone(s)
        opt.step(step=step, seed=2 ** 63 + 11, **hyper)
        torch.cuda.synchronize()
        _check_step(before, s, wd, eight, copies, hyper, step, 2 ** 63 + 11)
    opt.close()


def test_adamw_blocks_with_nothing_in_them_tiny_values_and_nan(cl):
    rng = np.random.default_rng(11)
    s = _adam_state(rng, [256 * 5 + 7], True, torch.float32, False)
    g = s["g"][0]
    s["m"][0].view(torch.uint8).zero_(); s["v"][0].view(torch.uint8).zero_()
    s["ms"][0].zero_(); s["vs"][0].zero_()
    g[:256] = 0.0                                  # nothing at all
    g[256:512] = 1e-38                             # squares vanish, magnitudes below the smallest scale
    g[512:768] *= 1e-15                            # (their squares are still above zero in fp32)
    g[512] = 3.0                                   # one large value: the others' codes round to 0 or 1
    g[800] = float("nan")                          # stays in its block
    before = _clone(s)
    opt = _make(cl, s, [0.0], True, False)
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
    opt.step(step=1, seed=5, **hyper)
    codes_v, m, p = _codes(s["v"][0]), s["m"][0].float(), s["p"][0]
    assert np.all(codes_v[:512] == 0) and float(s["vs"][0][0]) == 0.0 and float(s["vs"][0][1]) == 0.0
    assert np.all(codes_v[513:768] >= 1)           # a root that is not zero is not stored as zero
    nan = torch.isnan(p).cpu().numpy()
    assert nan.sum() == 1 and nan[800]
    assert torch.isnan(m[768:1024]).all() and not torch.isnan(m[1024:]).any() and not torch.isnan(m[:768]).any()
    keep = [k for k in range(256 * 5 + 7) if not 768 <= k < 1024]
    want = ref.adamw(before["p"][0].cpu().numpy(), before["g"][0].cpu().numpy(), _codes(before["m"][0]), _codes(before["v"][0]),
                     m_scale=before["ms"][0].cpu().numpy(), v_scale=before["vs"][0].cpu().numpy(), step=1, weight_decay=0.0, seed=5, **hyper)
    assert np.array_equal(_codes(s["m"][0])[keep], want[1][keep]) and np.array_equal(codes_v[keep], want[2][keep])
    assert np.array_equal(p.cpu().numpy()[keep], want[0][keep])


def test_adamw_8_bit_states_follow_a_change_of_the_gradients(cl):
    """Nearest rounding would leave v where it is; stochastic codes follow on average: after the gradients shrink to a
    third for 1500 steps the mean of v is within 10 % of the 32-bit state's."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    n = 1 << 16
    z = lambda dt=torch.float32: torch.zeros(n, dtype=dt, device=_dev())  # noqa: E731
    p8, p32, g = z(), z(), z()
    m32, v32 = z(), z()
    m8, v8 = z(torch.uint8).view(torch.float8_e4m3fn), z(torch.uint8).view(torch.float8_e4m3fn)
    ms, vs = torch.zeros(n // 256, device=_dev()), torch.zeros(n // 256, device=_dev())
    a = cl.AdamW([p8], [g], [m8], [v8], m_scales=[ms], v_scales=[vs])
    b = cl.AdamW([p32], [g], [m32], [v32])
    for t in range(1, 2001):
        g.normal_(generator=gen)
        g.mul_(1.0 if t <= 500 else 1 / 3)
        a.step(step=t, lr=1e-3, seed=3)
        b.step(step=t, lr=1e-3)
    v = (v8.float().view(-1, 256) * vs[:, None]).square().mean()
    assert abs(float(v / v32.mean()) - 1) < 0.1
    m = m8.float().view(-1, 256) * ms[:, None]
    assert float((m.view(-1) - m32).norm() / m32.norm()) < 0.2 and abs(float(m.mean() - m32.mean())) < 1e-3


def test_adamw_other_gradients_other_stream_and_refusals(cl):
    rng = np.random.default_rng(12)
    s = _adam_state(rng, [1000, 300], False, torch.float32, False)
    other = [t * 2 for t in s["g"]]
    hyper = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-6)
    opt = _make(cl, s, [0.0, 0.1], False, False)
    before = _clone(s)
    before["g"] = [t.clone() for t in other]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    opt.set_grads(other, stream=side)
    opt.step(step=3, stream=side, **hyper)
    side.synchronize()
    _check_step(before, s, [0.0, 0.1], False, False, hyper, 3, 0)
    for bad in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=float("nan")), dict(grad_scale=float("inf"))):
        with pytest.raises(cl.CleaveError) as e:
            opt.step(step=1, **{**hyper, **bad})
        assert e.value.code == -1
    with pytest.raises(ValueError):
        opt.step(step=0, **hyper)
    with pytest.raises(ValueError):
        opt.set_grads(other[:1])
    with pytest.raises(ValueError):
        cl.AdamW(s["p"], [t.to(torch.bfloat16) for t in s["g"][:1]] + s["g"][1:], s["m"], s["v"])
    empty = torch.zeros(0, device=_dev())
    cl.AdamW([empty], [empty], [empty], [empty]).step(step=1, lr=1.0)            # nothing to do


def test_adamw_tensors_without_a_copy(cl):
    rng = np.random.default_rng(13)
    s = _adam_state(rng, [700, 300], False, torch.float32, True)
    opt = cl.AdamW(s["p"], s["g"], s["m"], s["v"], copies=[None, s["w"][1]])
    hyper = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-6)
    before = _clone(s)
    opt.step(step=1, **hyper)
    _check_step(before, s, [0.0, 0.0], False, False, hyper, 1, 0)
    assert torch.all(s["w"][0] == 0) and torch.equal(s["w"][1], s["p"][1].to(torch.bfloat16))


# ---- norm -----------------------------------------------------------------------------------------------
NORM_SIZES = [(1, 1), (3, 7), (5, 8), (1, 4096), (33, 771), (4, 5120), (2, 16384), (2, 20001), (300, 64), (7, 1000), (2, 32768)]


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("x,res,y", [("bf16", "bf16", "bf16"), ("f32", None, "f32"), ("bf16", "f32", "e4m3"), ("f32", "bf16", "e4m3"), ("bf16", None, "bf16")])
def test_rmsnorm(cl, rows, cols, x, res, y):
    rng = np.random.default_rng(rows * 7 + cols)
    for pad in (0, 8, 3):
        xt = _strided(rng, rows, cols, DT[x], pad)
        rt = _strided(rng, rows, cols, DT[res], pad, 3.0) if res else None
        w = _rand(rng, cols, torch.float32 if pad == 0 else torch.bfloat16, 0.2) + 1 if pad != 3 else None
        yt = torch.zeros(rows, cols + pad, dtype=torch.float8_e4m3fn if y == "e4m3" else DT[y], device=_dev())[:, :cols]
        ht = torch.empty(rows, cols + pad, dtype=DT[res], device=_dev())[:, :cols] if res else None
        rstd = torch.empty(rows, device=_dev())
        scale = torch.empty(rows, device=_dev()) if y == "e4m3" else None
        cl.rmsnorm(xt, w, yt, residual=rt, h=ht, rstd=rstd, scale=scale, eps=1e-5)
        h64, y64, r64 = ref.rmsnorm(_f64(xt), _f64(rt), _f64(w), 1e-5)
        _close(rstd, r64, SUM * r64, "rstd")
        if res:
            _close(ht, h64, U * np.abs(h64), "h")
        if y == "e4m3":
            top = np.abs(y64).max(axis=1)
            _close(scale, top / 448, 2 * SUM * top / 448, "scale")
            q64 = y64 / _f64(scale)[:, None]
            err = np.abs(_f64(yt.float()) - q64)
            assert np.all(err <= 0.5 * ref.e4m3_step(q64) * (1 + 1e-3) + 2 * SUM * np.abs(q64))
        else:
            _close(yt, y64, 2 * SUM * np.abs(y64), "y")


def test_rmsnorm_in_place_zero_rows_nan_infinity_and_streams(cl):
    rng = np.random.default_rng(20)
    for cols in (512, 771):
        x, r = _rand(rng, (6, cols), torch.bfloat16), _rand(rng, (6, cols), torch.float32)
        x[2] = 0; r[2] = 0                                  # a row of zeros
        x[3, 5] = float("nan")
        x[4, 7] = float("inf")
        h64, y64, _ = ref.rmsnorm(_f64(x), _f64(r), None, 1e-5)
        fresh_h, y0, y1 = torch.empty_like(r), torch.empty_like(x), torch.empty_like(x)
        s0, q0 = torch.empty(6, device=_dev()), torch.zeros(6, cols, dtype=torch.float8_e4m3fn, device=_dev())
        cl.rmsnorm(x, None, y0, residual=r, h=fresh_h)
        cl.rmsnorm(x, None, q0, residual=r, scale=s0)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        cl.rmsnorm(x, None, y1, residual=r, h=r, stream=side)            # the sum replaces the residual
        side.synchronize()
        assert torch.equal(y0.view(torch.int16), y1.view(torch.int16)) and torch.equal(fresh_h.view(torch.int32), r.view(torch.int32))
        assert torch.all(y0[2] == 0) and float(s0[2]) == 0 and torch.all(q0[2].float() == 0)
        assert torch.isnan(y0[3]).all() and torch.isnan(s0[3])
        other = [c for c in range(cols) if c != 7]
        assert torch.isnan(y0[4, 7]) and torch.all(y0[4, other] == 0) and torch.isnan(s0[4])
        for i in (0, 1, 5):
            _close(y0[i:i + 1], y64[i:i + 1], 2 * SUM * np.abs(y64[i:i + 1]), f"row {i}")
    e = torch.empty(0, 8, dtype=torch.bfloat16, device=_dev())
    cl.rmsnorm(e, None, e.clone())
    big = torch.full((2, 256), 3e38, device=_dev())                       # h^2 overflows: rstd 0, y 0
    out = torch.empty_like(big)
    cl.rmsnorm(big, None, out)
    assert torch.all(out == 0)


@pytest.mark.parametrize("cols", [1, 8, 250, 4096, 20001])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_quantize_rows(cl, cols, dt):
    rng = np.random.default_rng(21)
    x = _rand(rng, (9, cols), DT[dt], 0.02)
    x[4] = 0
    q, s = torch.zeros(9, cols, dtype=torch.float8_e4m3fn, device=_dev()), torch.empty(9, device=_dev())
    cl.quantize_rows(x, q, s)
    x64 = _f64(x)
    _close(s, np.abs(x64).max(axis=1) / 448, 2 * U * np.abs(x64).max(axis=1) / 448, "scale")
    live = np.arange(9) != 4
    q64 = x64[live] / _f64(s)[live][:, None]
    assert np.all(np.abs(_f64(q.float())[live] - q64) <= 0.5 * ref.e4m3_step(q64) * (1 + 1e-3) + 4 * U * np.abs(q64))
    assert float(s[4]) == 0 and torch.all(q[4].float() == 0)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (5, 7), (400, 64), (33, 771), (1000, 1000), (6, 20001), (310, 5120), (3, 16384)])
@pytest.mark.parametrize("h,dy", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
def test_rmsnorm_backward(cl, rows, cols, h, dy):
    rng = np.random.default_rng(rows + cols)
    for pad in (0, 8, 1):
        ht, dyt = _strided(rng, rows, cols, DT[h], pad, 3.0), _strided(rng, rows, cols, DT[dy], pad)
        w = _rand(rng, cols, torch.float32 if pad == 0 else torch.bfloat16, 0.2) + 1 if pad != 1 else None
        dres = _strided(rng, rows, cols, DT[h], pad) if pad != 8 else None
        rstd = torch.rsqrt(ht.float().square().mean(1) + 1e-5)
        dx, dw = torch.empty(rows, cols + pad, dtype=DT[h], device=_dev())[:, :cols], torch.full((cols,), float("nan"), device=_dev())
        cl.rmsnorm_backward(dyt, ht, w, rstd, dx, dw, dres=dres)
        a = [_f64(t) for t in (dyt, ht, w, rstd, dres)]
        dx64, dw64 = ref.rmsnorm_backward(*a)
        q = np.abs(a[0] if a[2] is None else a[0] * a[2])
        xh = np.abs(a[1] * a[3][:, None])
        size = a[3][:, None] * (q + xh * np.mean(q * xh, axis=1, keepdims=True)) + (0 if dres is None else np.abs(a[4]))
        _close(dx, dx64, SUM * size, "dx")
        _close(dw, dw64, SUM * np.sum(np.abs(a[0]) * xh, axis=0), "dw")
        again, dx2 = torch.empty_like(dw), dx if dres is None else dres
        cl.rmsnorm_backward(dyt, ht, w, rstd, dx2, again, dres=dres)     # in place over dres; the same bits again
        assert torch.equal(again.view(torch.int32), dw.view(torch.int32)) and torch.equal(dx2, dx)


def test_rmsnorm_backward_without_rows_or_without_dw(cl):
    e = torch.empty(0, 40, device=_dev())
    dw = torch.ones(40, device=_dev())
    cl.rmsnorm_backward(e, e, None, torch.empty(0, device=_dev()), e, dw)
    assert torch.all(dw == 0)
    rng = np.random.default_rng(30)
    h, dy = _rand(rng, (9, 40), torch.float32), _rand(rng, (9, 40), torch.float32)
    rstd = torch.rsqrt(h.square().mean(1) + 1e-5)
    a, b = torch.empty_like(h), torch.empty_like(h)
    cl.rmsnorm_backward(dy, h, None, rstd, a, None)
    ws = torch.empty(cl.rmsnorm_backward_workspace(9, 40), dtype=torch.uint8, device=_dev())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    cl.rmsnorm_backward(dy, h, None, rstd, b, dw, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(a, b)
    with pytest.raises(ValueError):
        cl.rmsnorm_backward(dy, h, None, rstd, a, dw, workspace=ws[:8])


# ---- product with an epilogue -------------------------------------------------------------------------------
def _operands(rng, m, n, k, ta, tb, kind, pad, integer=True):
    """Stored A and B (rows a multiple of 16 elements apart) and their fp64 views as the product sees them."""
    dt = torch.float8_e4m3fn if kind == "e4m3" else torch.bfloat16

    def store(rows, cols):
        ld = -(-cols // 16) * 16 + pad
        v = rng.integers(-4, 5, size=(rows, ld)) if integer else rng.normal(size=(rows, ld))
        return torch.tensor(v, dtype=torch.float32).to(dt).to(_dev())[:, :cols]
    A, B = store(k, m) if ta else store(m, k), store(n, k) if tb else store(k, n)
    a, b = _f64(A.float()), _f64(B.float())
    return A, B, (a.T if ta else a), (b.T if tb else b)


LAYOUTS = [(False, False, "bf16"), (False, True, "bf16"), (True, False, "bf16"), (True, True, "bf16"), (False, True, "e4m3")]


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 4096, 512), (16, 512, 4096), (128, 128, 64), (129, 257, 65), (77, 33, 200), (300, 520, 1000),
                                   (8, 136, 3000), (260, 24, 72), (640, 1000, 130), (1, 8, 16384), (513, 769, 385),
                                   (4700, 1300, 200), (257, 20000, 72), (2500, 2500, 1100), (2600, 3080, 64), (1, 38000, 600)])
@pytest.mark.parametrize("ta,tb,kind", LAYOUTS)
def test_linear_integer_products_are_exact(cl, m, n, k, ta, tb, kind):
    """Integers in -4..4: every fp32 sum is exact, so every value has to be equal, in every layout and size."""
    rng = np.random.default_rng(m + n + k)
    A, B, a, b = _operands(rng, m, n, k, ta, tb, kind, 16 if m % 2 else 0)
    out = torch.full((m, n), float("nan"), device=_dev())
    cl.linear(A, B, out, transA=ta, transB=tb)
    assert cl.linear_status() == 0
    assert np.array_equal(_f64(out), a @ b)
    wide = torch.full((m, n + 5), 7.0, device=_dev())                     # padded rows: nothing outside C is written
    cl.linear(A, B, wide[:, :n], transA=ta, transB=tb, residual=out)
    assert np.array_equal(_f64(wide[:, :n]), 2 * (a @ b)) and torch.all(wide[:, n:] == 7.0)


@pytest.mark.parametrize("m,n,k", [(2500, 2048, 200), (2560, 2000, 72), (2560, 1930, 1100), (2800, 2304, 136), (75 * 256, 256, 130), (256, 19000, 640)])
@pytest.mark.parametrize("ta,tb,kind", LAYOUTS)
def test_linear_last_wave_of_large_products(cl, m, n, k, ta, tb, kind):
    """Tiles of 256 x 256 that do not divide over the GPU's 74 pairs of SMs: a few left over, many, ragged ones."""
    rng = np.random.default_rng(m + n + k)
    A, B, a, b = _operands(rng, m, n, k, ta, tb, kind, 0)
    want = a @ b
    for dt in (torch.float32, torch.bfloat16):
        out = torch.full((m, n), float("nan"), dtype=dt, device=_dev())
        z = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device=_dev())
        cl.linear(A, B, out, transA=ta, transB=tb, act="relu", z=z)
        assert cl.linear_status() == 0
        rounded = torch.tensor(want).to(_dev())
        assert torch.equal(z, rounded.to(torch.bfloat16))
        assert torch.equal(out, rounded.clamp(min=0).to(dt))


@pytest.mark.parametrize("m,n,k", [(10000, 200, 2050), (19100, 130, 72), (38000, 40, 130), (38000, 96, 640), (38000, 8, 64), (19000, 225, 1030)])
@pytest.mark.parametrize("ta,tb,kind", LAYOUTS)
def test_linear_by_pairs_with_narrow_tiles(cl, m, n, k, ta, tb, kind):
    """Products of many rows and fewer than 256 columns: a pair's tile is as wide as C (in steps of 32 columns)."""
    rng = np.random.default_rng(m + n + k)
    A, B, a, b = _operands(rng, m, n, k, ta, tb, kind, 0)
    want = torch.tensor(a @ b).to(_dev())
    for dt in (torch.float32, torch.bfloat16):
        out = torch.full((m, n + 3), 7.0, dtype=dt, device=_dev())
        z = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device=_dev())
        cl.linear(A, B, out[:, :n], transA=ta, transB=tb, act="relu", z=z)
        whole = torch.full((m, n), float("nan"), dtype=dt, device=_dev())
        cl.linear(A, B, whole, transA=ta, transB=tb, act="relu")
        assert cl.linear_status() == 0
        assert torch.equal(z, want.to(torch.bfloat16))
        assert torch.equal(whole, want.clamp(min=0).to(dt))
        assert torch.equal(out[:, :n], whole) and torch.all(out[:, n:] == 7.0)


@pytest.mark.parametrize("act", KINDS)
@pytest.mark.parametrize("kind,c,side", [("bf16", "bf16", "f32"), ("bf16", "f32", "bf16"), ("e4m3", "bf16", "bf16")])
@pytest.mark.parametrize("m,n,k", [(1, 72, 256), (200, 300, 320), (130, 129, 70), (16, 2048, 1024), (700, 512, 256), (3, 37993, 72), (130, 19008, 40)])
def test_linear_epilogue(cl, act, kind, c, side, m, n, k):
    rng = np.random.default_rng(m * n + k)
    A, B, a, b = _operands(rng, m, n, k, False, True, kind, 0, integer=False)
    sa = torch.tensor(rng.uniform(0.5, 1.5, size=m), dtype=torch.float32).to(_dev()) if kind == "e4m3" else None
    sb = torch.tensor(rng.uniform(0.02, 0.06, size=n), dtype=torch.float32).to(_dev())
    bias = _rand(rng, n, DT[side])
    mul, res = _rand(rng, (m, n), DT[side]), _rand(rng, (m, n), DT[c])
    z = torch.empty(m, n, dtype=DT[side], device=_dev())
    out = res.clone()
    for gate, add in ((mul, True), (None, True), (mul, False), (None, False)):
        out.copy_(res)
        cl.linear(A, B, out, transB=True, scale_a=sa, scale_b=sb, bias=bias, act=act, z=z, mul=gate, residual=out if add else None)
        assert cl.linear_status() == 0
        c64, z64 = ref.linear(a, b, scale_a=_f64(sa), scale_b=_f64(sb), bias=_f64(bias), kind=act, mul=_f64(gate), res=_f64(res) if add else None)
        # the products' terms in fp32, and the scales' and the bias's roundings
        size = (np.abs(a) @ np.abs(b)) * (1 if sa is None else _f64(sa)[:, None]) * _f64(sb) + np.abs(_f64(bias))
        zerr = SUM * size
        _close(z, z64, zerr, "z")
        # a slope of at most 1.13, then a few units of the activation's own arithmetic (its exponential's argument
        # is rounded at its own size)
        cerr = 1.13 * zerr + 32 * U * (1 + np.abs(z64)) * np.abs(z64)
        cerr = cerr if gate is None else cerr * np.abs(_f64(gate))
        _close(out, c64, cerr + 2 * U * (np.abs(c64) + (np.abs(_f64(res)) if add else 0)), "C")


def test_linear_nan_and_infinity_stay_in_their_rows_and_columns(cl):
    rng = np.random.default_rng(40)
    for m, n, k in ((150, 200, 128), (700, 600, 256)):
        A, B, a, b = _operands(rng, m, n, k, False, False, "bf16", 0)
        A[3, 5] = float("nan")
        B[7, 11] = float("inf")
        out = torch.empty(m, n, device=_dev())
        cl.linear(A, B, out)
        g = _f64(out)
        rows, cols = np.arange(m) != 3, np.arange(n) != 11
        assert np.isnan(g[3]).all() and np.array_equal(g[np.ix_(rows, cols)], (a @ b)[np.ix_(rows, cols)])
        assert not np.isfinite(g[rows][:, 11]).any()


# split form with 1, 2 and 4 CTAs a tile and with one row of tiles, pairs of CTAs
LONG_K = [(2048, 1280, 1900), (2048, 1280, 8192), (1100, 1500, 16384), (700, 900, 16400), (128, 20480, 8192), (1, 19200, 9000), (600, 1030, 4700), (4096, 2560, 8192)]


@pytest.mark.parametrize("m,n,k", LONG_K)
@pytest.mark.parametrize("ta,tb,kind", [(False, False, "bf16"), (True, False, "bf16"), (False, True, "e4m3")])
def test_linear_fp32_results_of_a_long_k_keep_their_accuracy(cl, m, n, k, ta, tb, kind):
    """Operands of one sign, so that what the tensor core cuts off adds up.  It adds 16 (E4M3: 32) products a step and may cut
    off a unit (2^-23) of the running sum; an accumulator takes 32 steps, whose running sums are half of the last
    one on average: 17 units of 2^-23.  The chunks' sums are rounded: half a unit of the running sum each, again half on
    average, and a few more in the cluster's sum.  (One accumulator over 8192 products: 9e-6, about three times the bound.)"""
    gen = torch.Generator(device=_dev()).manual_seed(m + n + k)
    dt = torch.float8_e4m3fn if kind == "e4m3" else torch.bfloat16

    def store(rows, cols):
        return (torch.rand(rows, -(-cols // 16) * 16, generator=gen, device=_dev()) + 0.5).to(dt)[:, :cols]
    A, B = store(k, m) if ta else store(m, k), store(n, k) if tb else store(k, n)
    a, b = (A.double().t() if ta else A.double()), (B.double().t() if tb else B.double())
    want = a @ b
    bound = 17 * 2.0 ** -23 + (k / 512 / 2 + 8) * 2.0 ** -24
    out, z = torch.full((m, n), float("nan"), device=_dev()), torch.full((m, n), float("nan"), device=_dev())
    cl.linear(A, B, out, transA=ta, transB=tb)
    assert cl.linear_status() == 0
    assert float((out.double() / want - 1).abs().max()) <= bound
    narrow = torch.empty(m, n, dtype=torch.bfloat16, device=_dev())
    cl.linear(A, B, narrow, transA=ta, transB=tb, act="relu", z=z)        # an fp32 z alone asks for it too
    assert torch.equal(z, out) and torch.equal(narrow, out.to(torch.bfloat16))


@pytest.mark.parametrize("m,n,k", [(300, 700, 5000), (1900, 1300, 1100), (1900, 1300, 4100), (1, 8, 4200), (129, 1, 9000), (100, 19100, 513), (1100, 1500, 3333)])
@pytest.mark.parametrize("ta,tb,kind", LAYOUTS)
def test_linear_handed_over_sums_are_whole(cl, m, n, k, ta, tb, kind):
    """Integers, exact in fp32: no chunk of K is lost or taken twice, whatever the number of chunks."""
    rng = np.random.default_rng(m + n + k)
    A, B, a, b = _operands(rng, m, n, k, ta, tb, kind, 0)
    out = torch.full((m, n + 4), 7.0, device=_dev())
    cl.linear(A, B, out[:, :n], transA=ta, transB=tb)
    assert cl.linear_status() == 0
    assert np.array_equal(_f64(out[:, :n]), a @ b) and torch.all(out[:, n:] == 7.0)


def test_linear_extreme_preactivations(cl):
    """Activations far out on either side: their limits, no NaN."""
    n = 64
    bias = torch.linspace(-1e4, 1e4, n, device=_dev())
    bias[0], bias[-1] = -1e30, 1e30
    A, B = torch.zeros(3, 8, dtype=torch.bfloat16, device=_dev()), torch.zeros(8, n, dtype=torch.bfloat16, device=_dev())
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        out = torch.empty(3, n, device=_dev())
        cl.linear(A, B, out, bias=bias, act=act)
        want = torch.clamp_min(bias, 0).expand(3, n)
        assert torch.allclose(out, want, rtol=1e-6, atol=0), act
        dz = torch.empty(3, n, device=_dev())
        cl.act_backward(torch.ones(3, n, device=_dev()), bias.expand(3, n).contiguous(), dz, act=act)
        assert torch.allclose(dz, (bias > 0).float().expand(3, n), rtol=1e-6, atol=1e-6), act


def _activation64(z, act):
    """Value, slope, and the size of the slope's terms, in 64 bits without cancellation on the negative side."""
    if act == "gelu":
        phi, bell = 0.5 * torch.special.erfc(-z * 0.5 ** 0.5), torch.exp(-0.5 * z * z) * (0.5 / np.pi) ** 0.5
        return z * phi, phi + z * bell, phi + z.abs() * bell
    u, du = (z, torch.ones_like(z)) if act == "silu" else (2 * (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3), 2 * (2 / np.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z))
    g, rest = torch.special.expit(u), torch.special.expit(-u)
    return z * g, g + z * g * rest * du, g + (z * g * rest * du).abs()


@pytest.mark.parametrize("act,low,units", [("gelu", -12.5, lambda z: 16 * (1 + z * z)), ("silu", -80.0, lambda z: 8 + 3 * z.abs()),
                                           ("gelu_tanh", -9.0, lambda z: 8 + 4 * 2 * (2 / np.pi) ** 0.5 * (z.abs() + 0.044715 * z.abs() ** 3))])
def test_activations_keep_their_digits_on_the_negative_side(cl, act, low, units):
    """Errors relative to the value itself, in fp32, for arguments put in through the bias.  GELU: the exponent -z^2 / 2 log2(e) takes
    two roundings and its constant's, which makes z^2 times 1.25 units; the polynomial (8.4e-8), its eight steps, the reciprocal
    (2 units, its effect at most doubled by the polynomial's slope) and the exponential (4 units) the rest.  The other
    two: gate = 1 / (1 + exp(-u)), u with at most four roundings of its own size, then exponential, sum and reciprocal."""
    n = 20000
    z = torch.cat([torch.linspace(low, 12.0, n - 200), -torch.logspace(-20, 0, 100), torch.logspace(-20, 0, 100)]).to(_dev())
    A, B = torch.zeros(2, 8, dtype=torch.bfloat16, device=_dev()), torch.zeros(8, n, dtype=torch.bfloat16, device=_dev())
    out = torch.empty(2, n, device=_dev())
    cl.linear(A, B, out, bias=z, act=act)
    value, slope, size = _activation64(z.double(), act)
    bound = units(z.double()) * U
    assert torch.all((out[1].double() - value).abs() <= (bound + U) * value.abs())
    for cols in (n, n - 1):                                   # the wide form and the one for any size
        zz, one = z[:cols].expand(2, cols).contiguous(), torch.ones(2, cols, device=_dev())
        dz, dmul = torch.empty_like(zz), torch.empty_like(zz)
        cl.act_backward(one, zz, dz, act=act, dmul=dmul)
        assert torch.all((dmul[1].double() - value[:cols]).abs() <= (bound + U)[:cols] * value[:cols].abs())
        # (1 - gate keeps only its absolute digits where the gate is close to 1, on the positive side: a unit of the factor)
        extra = 0 if act == "gelu" else 4 * U * (z[:cols].double().clamp_min(0) * (1 if act == "silu" else 2.0 + 0.3 * z[:cols].double() ** 2))
        assert torch.all((dz[1].double() - slope[:cols]).abs() <= (2 * bound + 4 * U)[:cols] * size[:cols] + extra)


def test_linear_repeats_its_bits_on_any_stream(cl):
    rng = np.random.default_rng(41)
    A, B, a, b = _operands(rng, 16, 1024, 4096, False, False, "bf16", 0, integer=False)
    first, second = torch.empty(16, 1024, device=_dev()), torch.empty(16, 1024, device=_dev())
    cl.linear(A, B, first)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        cl.linear(A, B, second, stream=side)
    assert cl.linear_status(side) == 0
    assert torch.equal(first.view(torch.int32), second.view(torch.int32))
    e = torch.empty(0, 4096, dtype=torch.bfloat16, device=_dev())
    cl.linear(e, B, torch.empty(0, 1024, device=_dev()))


@pytest.mark.parametrize("m,n,k", [(16, 512, 4096), (3000, 2048, 1024)])
def test_a_wait_that_runs_out_ends_the_product_in_order(cl, m, n, k):
    """With a limit of 0 the first wait that is not satisfied at once gives up: the kernel returns, the status says
    so once, and the next product is right."""
    rng = np.random.default_rng(42)
    A, B, a, b = _operands(rng, m, n, k, False, False, "bf16", 0)
    out = torch.zeros(m, n, device=_dev())
    assert cl.linear_status() == 0
    try:
        cl.ops.lib.cleave_linear_set_wait_limit_ns(0)
        cl.linear(A, B, out)
        assert cl.linear_status() == -7
    finally:
        cl.ops.lib.cleave_linear_set_wait_limit_ns(2_000_000_000)
    assert cl.linear_status() == 0
    cl.linear(A, B, out)
    assert cl.linear_status() == 0
    assert np.array_equal(_f64(out), a @ b)


@pytest.mark.parametrize("m,n,k", [(16, 512, 16384), (1900, 1300, 4096)])
def test_a_wait_that_runs_out_while_sums_are_handed_over(cl, m, n, k):
    """The same with accumulators that take turns (fp32 results of a long K)."""
    test_a_wait_that_runs_out_ends_the_product_in_order(cl, m, n, k)


# ---- the epilogue's backward ------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (65, 33), (1000, 72), (513, 1001), (64, 512), (5000, 8)])
@pytest.mark.parametrize("act", KINDS)
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_act_backward(cl, rows, cols, act, t):
    rng = np.random.default_rng(rows + cols)
    for pad in (0, 3):
        dy, z, mul = (_strided(rng, rows, cols, DT[t], pad, s) for s in (1.0, 2.0, 1.0))
        dz, dmul = (torch.empty(rows, cols + pad, dtype=DT[t], device=_dev())[:, :cols] for _ in range(2))
        db = torch.full((cols,), float("nan"), device=_dev())
        for gate in (mul, None):
            cl.act_backward(dy, z, dz, act=act, mul=gate, dmul=dmul, dbias=db)
            y64, z64, g64 = _f64(dy), _f64(z), _f64(gate)
            dz64, dmul64, db64 = ref.act_backward(y64, z64, act, g64)
            # the exponential's argument is rounded at its own size (up to 2 |z| (1 + z^2 / 20)); slopes are at most 1.13
            own = 32 * U * (1 + np.abs(z64)) ** 2 * np.abs(y64)
            err = own if gate is None else own * np.abs(g64)
            _close(dz, dz64, err, "dz")
            _close(dmul, dmul64, own * np.abs(z64), "dmul")
            _close(db, db64, err.sum(axis=0) + SUM * np.abs(dz64).sum(axis=0), "dbias")
        again = torch.empty_like(db)
        cl.act_backward(dy, z, None, act=act, dbias=again)                 # the bias gradient alone, the same bits
        assert torch.equal(again.view(torch.int32), db.view(torch.int32))
        kept = dz.clone()
        cl.act_backward(dy, z, z, act=act)                                 # over z's buffer
        assert torch.equal(z, kept)


def test_act_backward_without_rows_and_plain_column_sums(cl):
    e = torch.empty(0, 24, device=_dev())
    db = torch.ones(24, device=_dev())
    cl.act_backward(e, None, dbias=db)
    assert torch.all(db == 0)
    dy = torch.tensor(np.random.default_rng(50).integers(-8, 9, size=(2000, 24)), dtype=torch.float32).to(_dev())
    cl.act_backward(dy, None, dbias=db)
    assert torch.equal(db, dy.sum(0))                                       # integers: exact in any order
    ws = torch.empty(cl.act_backward_workspace(2000, 24), dtype=torch.uint8, device=_dev())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    cl.act_backward(dy, None, dbias=db, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(db, dy.sum(0))
    with pytest.raises(ValueError):
        cl.act_backward(dy, None, dbias=db, workspace=ws[:16])


@pytest.mark.parametrize("ty,tz,tm,tdz,tdm", [("f32", "bf16", "bf16", "bf16", "bf16"), ("bf16", "f32", "f32", "f32", "f32"), ("f32", "bf16", "f32", "f32", "bf16"),
                                              ("bf16", "f32", "bf16", "bf16", "f32")])
@pytest.mark.parametrize("rows,cols", [(7, 48), (300, 264), (1200, 40)])
def test_act_backward_of_mixed_types(cl, ty, tz, tm, tdz, tdm, rows, cols):
    rng = np.random.default_rng(rows + cols)
    dy, z, mul = _rand(rng, (rows, cols), DT[ty]), _rand(rng, (rows, cols), DT[tz], 2.0), _rand(rng, (rows, cols), DT[tm])
    dz, dmul, db = torch.empty(rows, cols, dtype=DT[tdz], device=_dev()), torch.empty(rows, cols, dtype=DT[tdm], device=_dev()), torch.empty(cols, device=_dev())
    for act in ("relu", "silu"):
        cl.act_backward(dy, z, dz, act=act, mul=mul, dmul=dmul, dbias=db)
        y64, z64, m64 = _f64(dy), _f64(z), _f64(mul)
        dz64, dmul64, _ = ref.act_backward(y64, z64, act, m64)
        own = 32 * U * (1 + np.abs(z64)) ** 2 * np.abs(y64)                # (as above)
        _close(dz, dz64, own * np.abs(m64), "dz")
        _close(dmul, dmul64, own * np.abs(z64), "dmul")
        _close(db, dz64.sum(axis=0), (own * np.abs(m64)).sum(axis=0) + SUM * np.abs(dz64).sum(axis=0), "dbias")


@pytest.mark.parametrize("rows", [1, 2, 16, 17, 33, 100, 128, 129, 255, 256, 257, 600, 1023, 1024, 1025, 1500])
def test_act_backward_column_sums_are_whole_whatever_the_bands(cl, rows):
    """Integers, exact in any order: rows that make one band, a cluster of up to eight, more; any alignment; no row lost."""
    rng = np.random.default_rng(51 + rows)
    for cols in (1, 8, 33, 256, 300, 1032):
        for dt in (torch.float32, torch.bfloat16):
            dy = torch.tensor(rng.integers(-8, 9, size=(rows, cols)), dtype=torch.float32).to(dt).to(_dev())
            z = torch.tensor(rng.integers(-1, 2, size=(rows, cols)), dtype=torch.float32).to(dt).to(_dev())
            db, dz = torch.full((cols + 2,), 7.0, device=_dev()), torch.empty_like(dy)
            cl.act_backward(dy, None, dbias=db[:cols])
            assert torch.equal(db[:cols], dy.float().sum(0)) and torch.all(db[cols:] == 7.0)
            cl.act_backward(dy, z, dz, act="relu", dbias=db[1:cols + 1])
            want = torch.where(z > 0, dy, torch.zeros_like(dy))
            assert torch.equal(dz, want) and torch.equal(db[1:cols + 1], want.float().sum(0)) and float(db[cols + 1]) == 7.0


# ---- one operator after another ------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols,ffn", [(3, 256, 512), (700, 768, 1536), (33, 130, 266)])
def test_chained_calls_see_what_the_one_before_wrote(cl, rows, cols, ffn):
    """Each call reads what the one before it writes, and buffers are written again two calls later; the same calls
    with the device idle in between, and replayed from a CUDA graph, leave the same bits."""
    rng = np.random.default_rng(rows)
    w1, w2 = _strided(rng, cols, ffn, torch.bfloat16, -ffn % 8, cols ** -0.5), _strided(rng, ffn, cols, torch.bfloat16, -cols % 8, ffn ** -0.5)
    norm, start, dy = _rand(rng, (cols,), torch.float32), _rand(rng, (rows, cols), torch.float32), _rand(rng, (rows, cols), torch.bfloat16)
    bf = lambda r, c: torch.empty(r, c + -c % 8, dtype=torch.bfloat16, device=_dev())[:, :c]  # noqa: E731 (operands' rows: 16 bytes)
    f32 = lambda *s: torch.empty(*s, device=_dev())  # noqa: E731
    stream = torch.cuda.Stream()
    spaces = [torch.empty(cl.rmsnorm_backward_workspace(rows, cols), dtype=torch.uint8, device=_dev()),
              torch.empty(cl.act_backward_workspace(rows, ffn), dtype=torch.uint8, device=_dev())]

    def buffers():
        return dict(h=start.clone(), y=bf(rows, cols), z=bf(rows, ffn), a=bf(rows, ffn), out=bf(rows, cols).zero_(), rstd=f32(rows), dz=bf(rows, ffn),
                    db=f32(ffn), da=bf(rows, ffn), dh=f32(rows, cols), dw=f32(cols), g=f32(rows, cols).zero_())

    def chain(t, between):
        for _ in range(3):
            for call in (lambda: cl.rmsnorm(t["out"], norm, t["y"], residual=t["h"], h=t["h"], rstd=t["rstd"], stream=stream),
                         lambda: cl.linear(t["y"], w1, t["a"], act="gelu_tanh", z=t["z"], stream=stream),
                         lambda: cl.linear(t["a"], w2, t["out"], stream=stream),
                         lambda: cl.linear(t["out"], w2, t["da"], transB=True, stream=stream),
                         lambda: cl.act_backward(t["da"], t["z"], t["dz"], act="gelu_tanh", dbias=t["db"], workspace=spaces[1], stream=stream),
                         lambda: cl.linear(t["dz"], w1, t["out"], transB=True, stream=stream),
                         lambda: cl.rmsnorm_backward(dy, t["h"], norm, t["rstd"], t["dh"], t["dw"], dres=t["g"], workspace=spaces[0], stream=stream),
                         lambda: cl.rmsnorm_backward(t["out"], t["h"], norm, t["rstd"], t["g"], t["dw"], dres=t["dh"], workspace=spaces[0], stream=stream)):
                call()
                between()

    slow, fast, replayed = buffers(), buffers(), buffers()
    torch.cuda.synchronize()
    chain(slow, torch.cuda.synchronize)
    chain(fast, lambda: None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        chain(replayed, lambda: None)
    graph.replay()
    torch.cuda.synchronize()
    for k, v in slow.items():
        assert torch.isfinite(v.float()).all(), k
        assert torch.equal(v, fast[k]), k
        assert torch.equal(v, replayed[k]), k


def test_workspaces_of_calls_on_another_stream_are_not_memory_in_use(cl):
    """A block of the workspace's size is freed on the current stream while work that reads and writes it is still
    queued there; calls on another stream that bring no workspace compute as ever, and so does the queued work."""
    rng = np.random.default_rng(60)
    rows, cols = 600, 1024
    h, dy = _rand(rng, (rows, cols), torch.float32), _rand(rng, (rows, cols), torch.float32)
    rstd = torch.rsqrt(h.square().mean(1) + 1e-5)
    dx, dw, want_dw = torch.empty_like(h), torch.zeros(cols, device=_dev()), torch.zeros(cols, device=_dev())
    db, want_db = torch.zeros(cols, device=_dev()), torch.zeros(cols, device=_dev())
    cl.rmsnorm_backward(dy, h, None, rstd, dx, want_dw)
    cl.act_backward(dy, None, dbias=want_db)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=_dev())
    for size, call, got, want in (
            (cl.rmsnorm_backward_workspace(rows, cols), lambda s: cl.rmsnorm_backward(dy, h, None, rstd, dx, dw, stream=s), dw, want_dw),
            (cl.act_backward_workspace(rows, cols), lambda s: cl.act_backward(dy, None, dbias=db, stream=s), db, want_db)):
        for stream in (side, side.cuda_stream):
            got.zero_()
            torch.cuda.synchronize()
            for _ in range(3):
                big @ big                                            # the current stream is busy for a few milliseconds
            block = torch.full((size // 4,), 3.0, device=_dev())
            kept = block + 1.0
            del block                                                # free for the current stream, whose work has not begun
            call(stream)
            torch.cuda.synchronize()
            assert torch.all(kept == 4.0) and torch.equal(got, want)
    # the workspaces' blocks belong to the launch's stream
    assert side.cuda_stream in {s["stream"] for s in torch.cuda.memory_snapshot()}
