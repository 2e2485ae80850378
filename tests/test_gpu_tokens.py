"""The operators on tokens and layer norm on the GPU against their 64-bit oracle.  Tolerances are the roundings of the stated
arithmetic: U = 2^-24 is half a unit of fp32, a bf16 result may be half a unit of its 8 significant bits (2^-8) off; a sum
of n terms that is split over lanes and warps is off by a modest multiple of U of its terms' magnitudes (64 U, as for sums
over lanes of up to 2^15 terms each); one that is added term by term by n U.  exp2 is the hardware's, 4 U of its result; an exponent t
that was rounded is off by U |t|, its power by as much relative to itself (times ln 2 and log2 e, which cancel)."""
import numpy as np
import pytest
import torch

from oracle import tokens as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SUM = 64 * U
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}
INF = float("inf")
LOW = {"bf16": float(torch.finfo(torch.bfloat16).min), "f32": float(torch.finfo(torch.float32).min)}


@pytest.fixture(scope="module")
def cl():
    import paper_2512_22142_b200 as cl
    return cl


def _dev():
    return torch.device("cuda:0")


def _put(a, dtype):
    return torch.tensor(a, dtype=torch.float32).to(dtype).to(_dev())


def _rand(rng, shape, dtype, scale=1.0):
    return _put(rng.normal(size=shape) * scale, dtype)


def _f64(t):
    return None if t is None else t.to(torch.float64).cpu().numpy()


def _lay(t, pad=0, shift=0):
    """The same matrix with rows `cols + pad` apart, beginning `shift` elements into an allocation; what lies between is 7."""
    rows, cols = t.shape
    store = torch.full((shift + max(rows, 1) * (cols + pad),), 7, dtype=t.dtype, device=t.device)
    view = store[shift:].view(max(rows, 1), cols + pad)[:rows, :cols]
    view.copy_(t)
    return view


def _room(rows, cols, dtype, pad=0, shift=0):
    """An output whose rows lie `cols + pad` apart, full of NaN, and the whole store with 7 behind each row."""
    store = torch.full((shift + max(rows, 1) * (cols + pad),), 7.0, dtype=torch.float32, device=_dev()).to(dtype)
    view = store[shift:].view(max(rows, 1), cols + pad)
    view[:, :cols] = float("nan") if dtype.is_floating_point else -7
    return view[:rows, :cols], view


def _untouched(view, cols):
    assert torch.all(view[:, cols:].float() == 7.0), "written behind a row"


def _close(got, want, tol, what=""):
    """|got - want| <= tol + the rounding of got's type; infinities and NaN in the same places."""
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    g, want = _f64(got), np.asarray(want, dtype=np.float64)
    want = np.where(np.abs(want) >= 2.0 ** 128 * (1 - 2.0 ** -25), np.copysign(INF, want), want)      # what fp32 rounds to infinity
    assert np.array_equal(np.isnan(g), np.isnan(want)), f"{what}: NaN"
    odd = ~np.isfinite(want)
    assert np.array_equal(g[odd & ~np.isnan(want)], want[odd & ~np.isnan(want)]) and np.isfinite(g[~odd]).all(), f"{what}: infinities"
    g, w, tol = g[~odd], want[~odd], np.broadcast_to(tol, want.shape)[~odd]
    bad = np.abs(g - w) - (tol + half * np.maximum(np.abs(w), np.abs(g)) * 1.001 + 1e-38)
    assert bad.max(initial=-1.0) <= 0, f"{what}: {bad.max():.3e} over"


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


# ---- embedding -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,vocab,cols", [(1, 1, 1), (1, 50, 4096), (64, 300, 256), (777, 100, 33), (5, 1000, 1001), (3000, 77, 8), (40, 70, 5120)])
@pytest.mark.parametrize("table,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("ids", ["i32", "i64"])
def test_embedding(cl, n, vocab, cols, table, out, ids):
    rng = np.random.default_rng(n + cols)
    tokens = rng.integers(0, vocab, size=n)
    tokens[rng.random(n) < 0.1] = -1
    if n > 20:
        tokens[3:7] = [-100, vocab, vocab + 5, 2 ** 40 if ids == "i64" else 2 ** 31 - 1]
        tokens[7] = -(2 ** 33) if ids == "i64" else -(2 ** 31)
    t, e = torch.tensor(tokens, dtype=DT[ids], device=_dev()), _rand(rng, (vocab, cols), DT[table])
    for pad, shift, scale in ((0, 0, 1.0), (3, 0, 2.5), (8, 1, -0.3)):
        y, whole = _room(n, cols, DT[out], pad, shift)
        cl.embedding(t, _lay(e, pad, shift), y, scale=scale)
        s = float(np.float32(scale))
        want = ref.embedding(tokens, _f64(e), s)
        _close(y, want, U * np.abs(want), "out")
        _untouched(whole, cols)
    cl.embedding(t[:0], e, torch.empty(0, cols, device=_dev()))


def test_embedding_of_a_large_table(cl):
    """Rows whose addresses pass 2^32 elements and bytes."""
    cols, vocab = 4096, (1 << 32) // 4096 + 5
    table = torch.empty(vocab, cols, dtype=torch.bfloat16, device=_dev())
    rows = [0, 1, vocab // 2, vocab - 2, vocab - 1]
    for r in rows:
        table[r] = r % 251
    y = torch.empty(len(rows), cols, dtype=torch.bfloat16, device=_dev())
    cl.embedding(torch.tensor(rows, device=_dev()), table, y)
    assert torch.equal(y, torch.tensor([r % 251 for r in rows], dtype=torch.bfloat16, device=_dev())[:, None].expand(-1, cols))
    dy = torch.ones(len(rows), cols, dtype=torch.bfloat16, device=_dev())
    cl.embedding_backward(dy, torch.tensor(rows, device=_dev()), table, scale=3.0, accumulate=True)
    assert torch.equal(table[rows], y + 3)
    cl.embedding_backward(dy, torch.tensor(rows, device=_dev()), table, scale=3.0)
    assert torch.all(table[rows] == 3) and float(table.sum(dtype=torch.float64)) == 3.0 * cols * len(rows)


def _spread_tokens(rng, n, vocab, how):
    if how == "one":
        return np.full(n, vocab // 2)
    if how == "each":
        return rng.permutation(np.arange(n) % vocab)
    if how == "sorted":
        return np.sort(rng.integers(0, vocab, size=n))
    t = np.minimum((np.exp(rng.random(n) * np.log(vocab + 1)) - 1).astype(np.int64), vocab - 1)     # frequency falls with the rank
    t[rng.random(n) < 0.1] = -1
    t[rng.random(n) < 0.02] = vocab
    return t


@pytest.mark.parametrize("n,vocab,cols", [(1, 1, 1), (1, 5000, 40), (15, 33, 8), (16, 40, 264), (17, 40, 1001), (4097, 500, 72), (30000, 3, 24), (2000, 70000, 16), (700, 31, 4104)])
@pytest.mark.parametrize("how", ["ranks", "one", "each", "sorted"])
def test_embedding_backward_is_whole(cl, n, vocab, cols, how):
    """Integers, exact in any order: no token is lost or taken twice, whatever their distribution; rows of absent tokens are zeros, or
    stay as they were."""
    rng = np.random.default_rng(n + vocab + cols)
    tokens = _spread_tokens(rng, n, vocab, how)
    for dy_t, dt_t, ids, pad, shift in (("bf16", "f32", "i64", 0, 0), ("f32", "f32", "i32", 3, 1), ("f32", "f32", "i64", 8, 0)):
        dy = _put(rng.integers(-8, 9, size=(n, cols)), DT[dy_t])
        t = torch.tensor(tokens, dtype=DT[ids], device=_dev())
        ok = (t >= 0) & (t < vocab)
        want = torch.zeros(vocab, cols, dtype=torch.float64, device=_dev()).index_add_(0, t[ok].long(), dy[ok].double()).float()
        dt, whole = _room(vocab, cols, DT[dt_t], pad, shift)
        cl.embedding_backward(_lay(dy, pad, shift), t, dt)
        assert torch.equal(dt, want)
        _untouched(whole, cols)
        before = _put(rng.integers(-8, 9, size=(vocab, cols)), DT[dt_t])
        dt.copy_(before)
        cl.embedding_backward(_lay(dy, pad, shift), t, dt, scale=2.0, accumulate=True)
        assert torch.equal(dt, before + 2 * want)
        _untouched(whole, cols)


@pytest.mark.parametrize("n,vocab,cols", [(3, 9, 100), (900, 40, 264), (5000, 2, 64), (1300, 4000, 129)])
@pytest.mark.parametrize("dy_t,dt_t", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_embedding_backward(cl, n, vocab, cols, dy_t, dt_t):
    rng = np.random.default_rng(n + cols)
    tokens = _spread_tokens(rng, n, vocab, "ranks")
    t, dy, before = torch.tensor(tokens, device=_dev()), _rand(rng, (n, cols), DT[dy_t]), _rand(rng, (vocab, cols), DT[dt_t])
    s = float(np.float32(1.7))
    for accumulate in (False, True):
        dt = before.clone()
        cl.embedding_backward(dy, t, dt, scale=1.7, accumulate=accumulate)
        want, size, count = ref.embedding_backward(_f64(dy), tokens, vocab, s, _f64(before) if accumulate else None)
        _close(dt, want, (count[:, None] + 4) * U * size, "dtable")
        again = before.clone()
        cl.embedding_backward(dy, t, again, scale=1.7, accumulate=accumulate)
        assert torch.equal(_bits(dt), _bits(again))                        # the same bits every time


def test_embedding_backward_without_tokens_and_with_padding_alone(cl):
    e = torch.empty(0, 24, device=_dev())
    for t, dy in ((torch.empty(0, dtype=torch.int64, device=_dev()), e), (torch.full((50,), -1, device=_dev()), torch.full((50, 24), float("nan"), device=_dev()))):
        dt = torch.ones(300, 24, device=_dev())
        cl.embedding_backward(dy, t, dt, accumulate=True)
        assert torch.all(dt == 1)
        cl.embedding_backward(dy, t, dt)
        assert torch.all(dt == 0)
    dt, dy = torch.ones(30, 8, device=_dev()), torch.full((4, 8), float("nan"), device=_dev())
    cl.embedding_backward(dy, torch.tensor([3, -1, 3, 99], device=_dev()), dt)
    assert torch.isnan(dt[3]).all() and float(dt.nan_to_num(0).sum()) == 0           # NaN stays in its token's row


# ---- layer norm ----------------------------------------------------------------------------------------
def _layernorm_tolerance(h, w, y, rstd, added):
    """What y may be off: the mean's sum, the root of the variance's sum (40 U: half of 64 U, and the root's own), the product and the
    sum with the bias, and what the residual's sum was rounded by."""
    mean_err = SUM * np.abs(h).mean(axis=1, keepdims=True) + U * np.abs(h).mean(axis=1, keepdims=True)
    scaled = np.abs(w) * rstd[:, None]
    xh = np.abs(h - h.mean(axis=1, keepdims=True)) * rstd[:, None]
    off = mean_err * rstd[:, None]                                          # of the normalised value, by the mean
    # (the variance is taken around the computed mean: off^2 more, relative to it)
    return scaled * (mean_err + (2 if added else 1) * U * np.abs(h)) + np.abs(w) * xh * (44 * U + off ** 2) + 3 * U * np.abs(y)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 8), (1, 4096), (33, 1000), (65, 768), (5, 1001), (2, 10000), (17, 2056), (700, 264), (3, 8192), (9, 5120), (1, 40000)])
@pytest.mark.parametrize("x,res,y", [("bf16", None, "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("bf16", "bf16", "e4m3"), ("f32", None, "e4m3"), ("f32", "bf16", "f32")])
def test_layernorm(cl, rows, cols, x, res, y):
    rng = np.random.default_rng(rows * 7 + cols)
    for pad, shift, wt in ((0, 0, "f32"), (3, 1, "bf16"), (8, 0, None)):
        xt = _lay(_rand(rng, (rows, cols), DT[x]) + 0.5, pad, shift)
        rt = None if res is None else _lay(_rand(rng, (rows, cols), DT[res], 3.0), pad, shift)
        w = None if wt is None else _rand(rng, cols, DT[wt], 0.2) + 1
        b = None if wt is None else _rand(rng, cols, DT[wt], 0.2)
        mean, rstd = torch.full((rows,), float("nan"), device=_dev()), torch.full((rows,), float("nan"), device=_dev())
        h, hw = _room(rows, cols, DT[res], pad, shift) if res else (None, None)
        h64, y64, m64, r64 = ref.layernorm(_f64(xt), _f64(rt), _f64(w), _f64(b), float(np.float32(1e-5)))
        tol = _layernorm_tolerance(h64, np.ones(cols) if w is None else _f64(w), y64, r64, res is not None)
        if y == "e4m3":
            store = torch.zeros(rows, cols + pad, dtype=torch.uint8, device=_dev())
            yt, scale = store.view(torch.float8_e4m3fn)[:, :cols], torch.full((rows,), float("nan"), device=_dev())
            cl.layernorm(xt, w, b, yt, residual=rt, h=h, mean=mean, rstd=rstd, scale=scale)
            top = np.abs(y64).max(axis=1)
            _close(scale, top / 448, tol.max(axis=1) / 448 + 2 * U * top / 448, "scale")
            s = _f64(scale)
            q = np.where(s[:, None] > 0, y64 / np.where(s > 0, s, 1)[:, None], 0.0)
            step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6))) - 3)
            got = _f64(yt.float())
            slack = np.where(s > 0, 1 / np.where(s > 0, s, 1), 0.0)[:, None] * tol + 4 * U * np.abs(q)
            assert (np.abs(got - q) <= step * 0.5 * 1.001 + slack).all()
            assert int(store[:, cols:].sum()) == 0
        else:
            yt, yw = _room(rows, cols, DT[y], pad, shift)
            cl.layernorm(xt, w, b, yt, residual=rt, h=h, mean=mean, rstd=rstd)
            _close(yt, y64, tol, "y")
            _untouched(yw, cols)
        if res:
            _close(h, h64, U * np.abs(h64), "h")
            _untouched(hw, cols)
        _close(mean, m64, (SUM + U) * np.abs(h64).mean(axis=1) + U * np.abs(m64), "mean")
        off = (SUM + U) * np.abs(h64).mean(axis=1) * r64
        _close(rstd, r64, (44 * U + off ** 2 + 2 * U * (np.abs(h64) * r64[:, None]).max(axis=1)) * r64, "rstd")


@pytest.mark.parametrize("cols", [8, 768, 1001, 4096, 5120])
def test_layernorm_of_rows_far_from_zero(cl, cols):
    """Values around 1000 with a spread of 1: a variance formed as a difference of squares would lose 1000^2 U."""
    rng = np.random.default_rng(cols)
    x = _put(rng.normal(size=(40, cols)) + 1000, torch.float32)
    x[:, 0] = -50000.0                                                      # and one column far out
    y, mean, rstd = torch.empty_like(x), torch.empty(40, device=_dev()), torch.empty(40, device=_dev())
    _, y64, m64, r64 = ref.layernorm(_f64(x), None, None, None, float(np.float32(1e-5)))
    cl.layernorm(x, None, None, y, mean=mean, rstd=rstd)
    _close(y, y64, _layernorm_tolerance(_f64(x), np.ones(cols), y64, r64, False), "y")
    x[:, 0] = 1001.0
    _, y64, m64, r64 = ref.layernorm(_f64(x), None, None, None, float(np.float32(1e-5)))
    cl.layernorm(x, None, None, y, mean=mean, rstd=rstd)
    _close(y, y64, _layernorm_tolerance(_f64(x), np.ones(cols), y64, r64, False), "y")
    # each variance's relative error: sums of squares of differences, which the mean's error changes in second order only
    assert (np.abs(_f64(rstd) / r64 - 1) <= 44 * U + (SUM * 1001 * r64) ** 2).all()


def test_layernorm_in_place_constant_rows_nan_and_no_rows(cl):
    rng = np.random.default_rng(5)
    for cols in (264, 1001, 4096, 20000):
        x, r = _rand(rng, (6, cols), torch.bfloat16), _rand(rng, (6, cols), torch.float32)
        x[1], r[1] = 2.0, 1.0                                               # a constant row: y is the bias
        x[3, 5] = float("nan")
        r[4, 7] = INF
        b, w = _rand(rng, cols, torch.float32), _rand(rng, cols, torch.float32)
        y, h, mean, rstd = (torch.empty(6, cols, device=_dev()), torch.empty_like(r), torch.empty(6, device=_dev()), torch.empty(6, device=_dev()))
        cl.layernorm(x, w, b, y, residual=r, h=h, mean=mean, rstd=rstd)
        assert torch.equal(y[1], b) and float(mean[1]) == 3.0 and abs(float(rstd[1]) * 1e-5 ** 0.5 - 1) < 1e-6
        assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all() and torch.isfinite(y[[0, 1, 2, 5]]).all()
        kept = r.clone()
        y2 = torch.empty_like(y)
        cl.layernorm(x, w, b, y2, residual=kept, h=kept)                    # h over the residual
        assert torch.equal(_bits(kept), _bits(h)) and torch.equal(_bits(y2), _bits(y))
        code, scale = torch.empty(6, cols, dtype=torch.float8_e4m3fn, device=_dev()), torch.empty(6, device=_dev())
        cl.layernorm(x, None, None, code, residual=r, scale=scale)
        assert float(scale[1]) == 0 and not code[1].float().any() and torch.isnan(scale[3]) and torch.isnan(scale[4])
        e = torch.empty(0, cols, device=_dev())
        cl.layernorm(e, None, None, e)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 8), (1, 4096), (300, 768), (5, 1001), (2, 10000), (33, 2056), (700, 264), (3, 8192), (310, 5120), (2, 33000)])
@pytest.mark.parametrize("dy_t,h_t", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
def test_layernorm_backward(cl, rows, cols, dy_t, h_t):
    rng = np.random.default_rng(rows + cols)
    for pad, shift, with_res, wt in ((0, 0, True, "f32"), (3, 1, False, "bf16"), (8, 0, True, None)):
        h, dy = _lay(_rand(rng, (rows, cols), DT[h_t], 2.0) + 0.5, pad, shift), _lay(_rand(rng, (rows, cols), DT[dy_t]), pad, shift)
        dres = _lay(_rand(rng, (rows, cols), DT[h_t]), pad, shift) if with_res else None
        w = None if wt is None else _rand(rng, cols, DT[wt], 0.2) + 1
        mean = h.float().mean(1)
        rstd = torch.rsqrt((h.float() - mean[:, None]).square().mean(1) + 1e-5)
        dx, whole = _room(rows, cols, DT[h_t], pad, shift)
        dw, db = torch.full((cols,), float("nan"), device=_dev()), torch.full((cols,), float("nan"), device=_dev())
        cl.layernorm_backward(dy, h, w, mean, rstd, dx, dw, db, dres=dres)
        h64, dy64, m64, r64 = _f64(h), _f64(dy), _f64(mean), _f64(rstd)
        w64 = np.ones(cols) if w is None else _f64(w)
        dx64, dw64, db64 = ref.layernorm_backward(dy64, h64, w64, m64, r64, _f64(dres))
        # xh: one rounding of the difference (which is that of its larger operand when they are far apart), one of the product
        xh = np.abs(h64 - m64[:, None]) * r64[:, None]
        xerr = 2 * U * xh + U * np.abs(h64 - m64[:, None]) * r64[:, None]
        q = np.abs(dy64 * w64)
        mean_qx, mean_q = (q * xh).mean(axis=1, keepdims=True), q.mean(axis=1, keepdims=True)
        tol = r64[:, None] * (4 * U * q + (SUM + 4 * U) * mean_q + xh * ((SUM + 8 * U) * mean_qx) + xerr * mean_qx + 4 * U * xh * mean_qx)
        tol = tol + 2 * U * (0 if dres is None else np.abs(_f64(dres))) + 2 * U * np.abs(dx64)
        _close(dx, dx64, tol, "dx")
        _untouched(whole, cols)
        _close(dw, dw64, (SUM + 4 * U) * (np.abs(dy64) * xh).sum(axis=0), "dw")
        _close(db, db64, SUM * np.abs(dy64).sum(axis=0), "db")
        again = torch.empty_like(db)
        cl.layernorm_backward(dy, h, w, mean, rstd, dx, None, again, dres=dres)          # one of the two, the same bits
        assert torch.equal(_bits(again), _bits(db))
        cl.layernorm_backward(dy, h, w, mean, rstd, dx, again, None, dres=dres)
        assert torch.equal(_bits(again), _bits(dw))
        if with_res:
            kept = dx.clone()
            cl.layernorm_backward(dy, h, w, mean, rstd, dres, dres=dres)                 # over dres, without sums
            assert torch.equal(_bits(dres), _bits(kept))


@pytest.mark.parametrize("rows", [1, 2, 31, 147, 148, 149, 295, 297, 600, 1500])
def test_layernorm_backward_column_sums_are_whole(cl, rows):
    """Integers, exact in any order."""
    rng = np.random.default_rng(rows)
    for cols in (1, 8, 33, 1032, 5128):
        dy, h = (_put(rng.integers(-4, 5, size=(rows, cols)), torch.bfloat16) for _ in range(2))
        one, zero = torch.ones(rows, device=_dev()), torch.zeros(rows, device=_dev())
        dx, dw, db = torch.empty_like(h), torch.full((cols + 1,), 7.0, device=_dev()), torch.full((cols + 1,), 7.0, device=_dev())
        cl.layernorm_backward(dy, h, None, zero, one, dx, dw[:cols], db[:cols])
        assert torch.equal(dw[:cols], (dy.float() * h.float()).sum(0)) and torch.equal(db[:cols], dy.float().sum(0))
        assert float(dw[cols]) == 7.0 and float(db[cols]) == 7.0
    e, dw, db = torch.empty(0, 24, device=_dev()), torch.ones(24, device=_dev()), torch.ones(24, device=_dev())
    v = torch.empty(0, device=_dev())
    cl.layernorm_backward(e, e, None, v, v, e, dw, db)
    assert not dw.any() and not db.any()


# ---- log probabilities -----------------------------------------------------------------------------------
def _scores(rng, rows, vocab, dtype, special=True):
    """Scores with a spread of 3, some masked, many of equal value in bf16; the last rows are special ones."""
    x = rng.normal(size=(rows, vocab)) * 3
    x[:, rng.random(vocab) < 0.05] = -INF
    x[:, 0] = 1.0
    x = torch.tensor(x, dtype=torch.float32).to(DT[dtype])
    if special:
        low = LOW[dtype]
        make = [lambda r: r.fill_(-INF), lambda r: r.fill_(low), lambda r: r.fill_(low)[vocab // 2].fill_(2.0), lambda r: r.fill_(0.0)[::2].fill_(-0.0),
                lambda r: r[vocab // 3].fill_(float("nan")), lambda r: r[vocab // 2].fill_(INF), lambda r: r.fill_(-INF)[vocab - 1].fill_(-5.0),
                lambda r: r.add_(300.0), lambda r: r.copy_(torch.linspace(-80, 80, vocab)), lambda r: r.copy_(torch.linspace(40, -40, vocab))]
        for i, f in enumerate(make):
            if i < rows - 1:
                f(x[rows - 1 - i])
    return x.to(_dev())


def _row_spread(x64, scale):
    """Per row: the sums over p of |d| and d^2, d = scale (x - largest), and |scale largest| (0 where there is no softmax)."""
    ed, ed2, top = (np.zeros(len(x64)) for _ in range(3))
    for i, r in enumerate(x64):
        lp, lse = ref.log_softmax(r, scale)
        if np.isfinite(lse):
            p, d = np.exp(lp), np.where(np.isfinite(r), scale * (r - r.max()), 0.0)
            ed[i], ed2[i], top[i] = (p * np.abs(d)).sum(), (p * d * d).sum(), abs(scale * r.max())
    return ed, ed2, top


def _statistics_tolerance(x64, scale):
    """(of lse, of entropy): a term e^d is off by (4 + 3 |d|) U relative to itself, its sum by 64 U more; lse adds the logarithm's
    rounding and its own at the size of scale * largest; entropy is log(sum) + sum(e |d|) / sum with the same terms."""
    ed, ed2, top = _row_spread(x64, scale)
    sum_err = SUM + (4 + 3 * ed) * U
    lse = sum_err + 4 * U * (top + np.log(x64.shape[1] + 1))
    return lse, 2 * sum_err * (1 + ed) + (8 * ed + 3 * ed2) * U + 4 * U * (np.log(x64.shape[1] + 1) + ed)


SHAPES = [(1, 1), (12, 2), (12, 7), (12, 8), (13, 33), (14, 255), (15, 1000), (16, 4097), (13, 20011), (1, 128000), (300, 520), (12, 50304)]


@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("x_t,ids,scale", [("bf16", "i64", 1.0), ("f32", "i32", 1.0), ("f32", "i64", 0.5), ("bf16", "i32", 1.7)])
def test_token_logprobs(cl, rows, vocab, x_t, ids, scale):
    rng = np.random.default_rng(rows + vocab)
    x = _scores(rng, rows, vocab, x_t, rows > 1)
    tokens = rng.integers(0, vocab, size=rows)
    tokens[rng.random(rows) < 0.1] = -100
    if rows > 2:
        tokens[:3] = [0, vocab - 1, vocab]
    t = torch.tensor(tokens, dtype=DT[ids], device=_dev())
    s = float(np.float32(scale))
    x64 = _f64(x)
    lse_tol, h_tol = _statistics_tolerance(x64, s)
    for pad, shift, top in ((0, 0, min(vocab, 5)), (3, 1, 0), (8, 0, min(vocab, 64)), (1, 3, 1)):
        f = lambda: torch.full((rows,), float("nan"), device=_dev())  # noqa: E731
        logp, lse, entropy = f(), f(), f()
        tv, tvw = _room(rows, top, torch.float32, 2) if top else (None, None)
        ti, tiw = _room(rows, top, torch.int32, 2) if top else (None, None)
        cl.token_logprobs(_lay(x, pad, shift), t, logp, lse=lse, entropy=entropy, top_values=tv, top_index=ti, scale=scale)
        w_logp, w_lse, w_h, w_tv, w_ti = ref.logprobs(x64, tokens, s, top)
        _close(lse, w_lse, lse_tol, "lse")
        _close(entropy, w_h, h_tol, "entropy")
        own = np.where((tokens >= 0) & (tokens < vocab), x64[np.arange(rows), np.clip(tokens, 0, vocab - 1)], 0.0)
        with np.errstate(invalid="ignore"):
            _close(logp, w_logp, lse_tol + np.where(np.isfinite(own), 3 * U * np.abs(s * own), 0.0), "logp")
            if top:
                assert np.array_equal(ti.cpu().numpy(), w_ti)
                picked = np.take_along_axis(x64, w_ti, 1)
                _close(tv, w_tv, lse_tol[:, None] + np.where(np.isfinite(picked), 3 * U * np.abs(s * picked), 0.0), "top values")
                _untouched(tvw, top)
                _untouched(tiw, top)


def test_token_logprobs_of_what_is_asked_for_alone(cl):
    """Each output without the others: the same bits."""
    rng = np.random.default_rng(9)
    for vocab in (300, 4097, 50257):
        x, t = _scores(rng, 14, vocab, "bf16"), torch.tensor(rng.integers(0, vocab, size=14), device=_dev())
        f = lambda: torch.full((14,), float("nan"), device=_dev())  # noqa: E731
        logp, lse, h, tv, ti = f(), f(), f(), torch.empty(14, 9, device=_dev()), torch.empty(14, 9, dtype=torch.int32, device=_dev())
        cl.token_logprobs(x, t, logp, lse=lse, entropy=h, top_values=tv, top_index=ti)
        for name, like in (("lse", lse), ("entropy", h), ("top_values", tv), ("top_index", ti)):
            got = torch.empty_like(like)
            cl.token_logprobs(x, None, None, **{name: got})
            assert torch.equal(_bits(got), _bits(like)), name
        got = f()
        cl.token_logprobs(x, t, got)
        assert torch.equal(_bits(got), _bits(logp))


@pytest.mark.parametrize("x_t", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [64, 700, 5000, 50257, 128000])
def test_top_places_of_adversarial_rows(cl, x_t, vocab):
    """Rows in which every place is better than all before it, equal values by the thousand, and few different ones."""
    rng = np.random.default_rng(vocab)
    rows = [np.arange(vocab) / vocab, -np.arange(vocab) / vocab, np.zeros(vocab), rng.integers(0, 3, size=vocab), np.where(np.arange(vocab) % 97 == 5, 2.0, -1.0),
            np.where(np.arange(vocab) >= vocab - 40, 1.0, 0.0), np.tile(np.arange(16), vocab // 16 + 1)[:vocab]]
    x = _put(np.array(rows, dtype=np.float64), DT[x_t])
    for top in (1, 20, 64):
        ti, tv = torch.full((len(rows), top), -1, dtype=torch.int32, device=_dev()), torch.empty(len(rows), top, device=_dev())
        cl.token_logprobs(x, top_values=tv, top_index=ti)
        want = np.array([ref.top_places(r, top) for r in _f64(x)])
        assert np.array_equal(ti.cpu().numpy(), want), top


@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("x_t,dx_t,scale", [("bf16", "bf16", 1.0), ("f32", "f32", 0.5), ("bf16", "f32", 1.7), ("f32", "bf16", 1.0)])
def test_token_logprobs_backward(cl, rows, vocab, x_t, dx_t, scale):
    rng = np.random.default_rng(rows + vocab)
    x = _scores(rng, rows, vocab, x_t, rows > 1)
    tokens = rng.integers(0, vocab, size=rows)
    tokens[rng.random(rows) < 0.1] = -100
    t = torch.tensor(tokens, device=_dev())
    s, x64 = float(np.float32(scale)), _f64(x)
    _, lse64, h64, _, _ = ref.logprobs(x64, tokens, s)
    lse, h = _put(lse64, torch.float32), _put(h64, torch.float32)
    up, dz, dh = (_rand(rng, rows, torch.float32) for _ in range(3))
    if rows > 11:
        up[0] = dz[0] = dh[0] = 0.0                                         # nothing asked: zeros
    for pad, shift, args in ((0, 0, dict(dlogp=up)), (3, 1, dict(dlogp=up, dlse=dz, dentropy=dh, entropy=h)), (8, 0, dict(dlse=dz)), (1, 2, dict(dentropy=dh, entropy=h))):
        dx, whole = _room(rows, vocab, DT[dx_t], pad, shift if dx_t == x_t else 0)
        kept = _lay(x, pad, shift)
        cl.token_logprobs_backward(kept, t if "dlogp" in args else None, lse, dx, scale=scale, **args)
        a = {k: _f64(v) for k, v in args.items()}
        with np.errstate(invalid="ignore"):
            want, size = ref.logprobs_backward(x64, tokens, _f64(lse), s, a.get("dlogp"), a.get("dlse"), a.get("dentropy"), a.get("entropy"))
            far = np.where(np.isfinite(x64) & np.isfinite(lse64)[:, None], np.abs(s * x64 - _f64(lse)[:, None]), 0.0)
            far = np.where(far > 200, 0.0, far)                             # (p is 0 there)
            # p: its exponent's two roundings and exp2's own; the factors' sums and products.  A p below 2^-126 is taken as 0, which
            # leaves out as much times the factor; |log p| is below 90 where p is not (and its own last place is 0.01)
            gone = 2.0 ** -126 * s * (np.abs(a.get("dlogp", np.zeros(rows))) + np.abs(a.get("dlse", np.zeros(rows))) +
                                      np.abs(a.get("dentropy", np.zeros(rows))) * (90 + np.abs(np.nan_to_num(_f64(h)))))
            _close(dx, want, np.where(np.isfinite(size), size * (3 * far + 16) * U, 0.0) + 1.02 * gone[:, None], "dx")
        _untouched(whole, vocab)
        if dx_t == x_t:
            cl.token_logprobs_backward(kept, t if "dlogp" in args else None, lse, kept, scale=scale, **args)      # over the scores
            nan = torch.isnan(dx)
            assert torch.equal(torch.isnan(kept), nan) and torch.equal(_bits(kept.masked_fill(nan, 0)), _bits(dx.masked_fill(nan, 0)))


def test_gradients_of_a_row_sum_to_what_lse_asks(cl):
    """Against differences of the forward pass in the direction of a random vector, in fp32."""
    rng = np.random.default_rng(12)
    x, t = _rand(rng, (30, 1003), torch.float32, 2.0), torch.tensor(rng.integers(0, 1003, size=30), device=_dev())
    v = _rand(rng, (30, 1003), torch.float32)
    f = lambda: torch.empty(30, device=_dev())  # noqa: E731
    logp, lse, h, dx = f(), f(), f(), torch.empty_like(x)
    cl.token_logprobs(x, t, logp, lse=lse, entropy=h, scale=0.7)
    up, z, e = (_rand(rng, 30, torch.float32) for _ in range(3))
    cl.token_logprobs_backward(x, t, lse, dx, dlogp=up, dlse=z, dentropy=e, entropy=h, scale=0.7)
    step, ends = 2.0 ** -6, []
    for sign in (1, -1):
        a, b, c = f(), f(), f()
        cl.token_logprobs(x + sign * step * v, t, a, lse=b, entropy=c, scale=0.7)
        ends.append(a.double() * up + b.double() * z + c.double() * e)
    slope = (ends[0] - ends[1]) / (2 * step)
    # the third derivative's share (step^2 / 6 of terms of size |v|^3 0.34) and the outputs' roundings over the step
    assert torch.allclose((dx.double() * v).sum(1), slope, rtol=2e-3, atol=3e-3)


# ---- distillation ------------------------------------------------------------------------------------------
def _teacher(rng, rows, vocab, k):
    index = np.array([rng.choice(vocab, size=k, replace=k > vocab) for _ in range(rows)])
    values = rng.normal(size=(rows, k)) * 2 - 3
    index[rng.random((rows, k)) < 0.05] = -1
    values[rng.random((rows, k)) < 0.05] = -INF
    if rows > 4:
        index[0] = -1                                                       # nothing to learn
        values[1] = -INF
        index[2] = index[2, 0]                                              # one place, k times
        index[3, : k // 2] = index[3, k - k // 2:][: k // 2]                # places that occur twice
        index[4, 0] = vocab
    return index, values


@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (16, 40, 7), (18, 1000, 64), (17, 4097, 256), (16, 20011, 33), (300, 520, 5), (2, 128000, 100), (20, 50304, 128)])
@pytest.mark.parametrize("x_t,dx_t,t_t,ids,normalize,scale", [("bf16", "bf16", "bf16", "i32", True, 0.5), ("f32", "f32", "f32", "i64", False, 1.0), ("f32", "bf16", "bf16", "i64", True, 1.0),
                                                              ("bf16", "f32", "f32", "i32", False, 1.3)])
def test_distill(cl, rows, vocab, k, x_t, dx_t, t_t, ids, normalize, scale):
    rng = np.random.default_rng(rows + vocab + k)
    x = _scores(rng, rows, vocab, x_t, False)
    if rows > 4:
        x[5].fill_(-INF)
        x[6, vocab // 2] = float("nan")
        x[7].fill_(LOW[x_t])
        x[0, 0] = float("nan")                                              # in a padded row: it does not matter
    index, values = _teacher(rng, rows, vocab, k)
    it, vt = torch.tensor(index, dtype=DT[ids], device=_dev()), torch.tensor(values, dtype=torch.float32).to(DT[t_t]).to(_dev())
    s, x64, v64 = float(np.float32(scale)), _f64(x), _f64(vt)
    dloss = _rand(rng, rows, torch.float32)
    if rows > 12:
        dloss[11] = 0.0
    with np.errstate(invalid="ignore"):
        w_loss, w_lse, size = ref.distill(x64, index, v64, s, normalize)
    lse_tol, _ = _statistics_tolerance(x64, s)
    # q: its exponent (the value less the largest, and the sum's 64 U), times a logarithm with the same error
    spread = np.array([np.abs(s * np.where(np.isfinite(v), v, 0)).max(initial=0) for v in v64])
    q_err = SUM + (4 + 6 * spread) * U
    for pad, shift in ((0, 0), (3, 1), (8, 0)):
        loss, lse = torch.full((rows,), float("nan"), device=_dev()), torch.full((rows,), float("nan"), device=_dev())
        xs, ixs, vs = _lay(x, pad, shift), _lay(it, pad), _lay(vt, pad, shift)
        cl.distill(xs, ixs, vs, loss, lse=lse, scale=scale, normalize=normalize)
        total = np.array([ref.teacher(i, v, vocab, s, normalize)[0].sum() for i, v in zip(index, v64)])
        with np.errstate(invalid="ignore"):
            biggest = np.array([np.abs(s * r[np.isfinite(r)]).max(initial=0) for r in x64])
            _close(loss, w_loss, np.where(np.isfinite(size), size, 0) * (q_err + 4 * U) + total * (lse_tol + q_err + 4 * U * biggest), "loss")
        _close(lse, w_lse, lse_tol, "lse")
        alone = torch.empty_like(loss)
        cl.distill(xs, ixs, vs, alone, scale=scale, normalize=normalize)
        assert torch.equal(_bits(alone), _bits(loss))
        dx, whole = _room(rows, vocab, DT[dx_t], pad, shift if dx_t == x_t else 0)
        given = _put(w_lse, torch.float32)
        cl.distill_backward(xs, ixs, vs, given, dloss, dx, scale=scale, normalize=normalize)
        with np.errstate(invalid="ignore"):
            want, terms = ref.distill_backward(x64, index, v64, _f64(given), _f64(dloss), s, normalize)
            far = np.where(np.isfinite(x64) & np.isfinite(w_lse)[:, None], np.abs(s * x64 - _f64(given)[:, None]), 0.0)
            far = np.where(far > 200, 0.0, far)
            _close(dx, want, np.where(np.isfinite(terms), terms, 0) * ((3 * far + 16) * U + q_err[:, None]) + 1e-37, "dx")
        _untouched(whole, vocab)
        if dx_t == x_t:
            cl.distill_backward(xs, ixs, vs, given, dloss, xs, scale=scale, normalize=normalize)                  # over the scores
            nan = torch.isnan(dx)
            assert torch.equal(torch.isnan(xs), nan) and torch.equal(_bits(xs.masked_fill(nan, 0)), _bits(dx.masked_fill(nan, 0)))


# ---- streams, graphs, no rows ---------------------------------------------------------------------------------
def test_no_rows(cl):
    e, v, t = torch.empty(0, 30, device=_dev()), torch.empty(0, device=_dev()), torch.empty(0, dtype=torch.int64, device=_dev())
    i, q = torch.empty(0, 4, dtype=torch.int32, device=_dev()), torch.empty(0, 4, device=_dev())
    cl.token_logprobs(e, t, v, lse=v, entropy=v, top_values=q, top_index=i)
    cl.token_logprobs_backward(e, t, v, e, dlogp=v)
    cl.distill(e, i, q, v, lse=v)
    cl.distill_backward(e, i, q, v, v, e)
    torch.cuda.synchronize()


def test_refusals_reach_the_caller(cl):
    x, v = torch.zeros(2, 10, device=_dev()), torch.zeros(2, device=_dev())
    t, i = torch.zeros(2, dtype=torch.int64, device=_dev()), torch.zeros(2, 300, dtype=torch.int32, device=_dev())
    for call in (lambda: cl.token_logprobs(x, t, v, scale=0.0), lambda: cl.token_logprobs(x, t, None), lambda: cl.token_logprobs(x, top_index=i[:, :11]),
                 lambda: cl.token_logprobs(torch.zeros(2, 100, device=_dev()), top_index=i[:, :65]), lambda: cl.token_logprobs_backward(x, t, v, x),
                 lambda: cl.distill(x, i, torch.zeros(2, 300, device=_dev()), v), lambda: cl.distill(x, i[:, :0], x[:, :0], v), lambda: cl.layernorm(x, None, None, x, eps=-1.0),
                 lambda: cl.embedding(t, x, x, scale=float("nan")), lambda: cl.layernorm(x, None, None, x, h=torch.zeros_like(x))):
        with pytest.raises(cl.CleaveError):
            call()


@pytest.mark.parametrize("rows,vocab,cols", [(3, 500, 256), (700, 4000, 768), (33, 1003, 130)])
def test_chained_calls_see_what_the_one_before_wrote(cl, rows, vocab, cols):
    """A training step's calls, each reading what the one before it wrote and buffers written again in the next round; the same
    calls with the device idle in between, and replayed from a CUDA graph, leave the same bits."""
    rng = np.random.default_rng(rows)
    tokens = torch.tensor(_spread_tokens(rng, rows, vocab, "ranks"), device=_dev())
    w, b = _rand(rng, cols, torch.float32, 0.1) + 1, _rand(rng, cols, torch.float32)
    table = _rand(rng, (vocab, cols), torch.float32)
    # operands of products: rows of whole 16 bytes
    even = lambda r, c: torch.zeros(r, c + -c % 8, dtype=torch.bfloat16, device=_dev())[:, :c]  # noqa: E731
    head = even(vocab, cols)
    head.copy_(table)
    index = torch.tensor(rng.integers(0, vocab, size=(rows, 12)), dtype=torch.int32, device=_dev())
    values, dloss = _rand(rng, (rows, 12), torch.float32), torch.full((rows,), 1.0 / rows, device=_dev())
    stream = torch.cuda.Stream()
    spaces = [torch.empty(cl.embedding_backward_workspace(rows, vocab, cols), dtype=torch.uint8, device=_dev()),
              torch.empty(cl.layernorm_backward_workspace(rows, cols), dtype=torch.uint8, device=_dev())]
    f32 = lambda *s: torch.zeros(*s, device=_dev())  # noqa: E731

    def buffers():
        return dict(e=table.clone(), x=even(rows, cols), h=f32(rows, cols), y=even(rows, cols), mean=f32(rows), rstd=f32(rows), z=even(rows, vocab), logp=f32(rows), lse=f32(rows), H=f32(rows),
                    dz=even(rows, vocab), dy=even(rows, cols), dh=f32(rows, cols), dw=f32(cols), db=f32(cols), dt=f32(vocab, cols), ti=torch.zeros(rows, 4, dtype=torch.int32, device=_dev()),
                    loss=f32(rows))

    def chain(t, between):
        for i in range(3):
            calls = [lambda: cl.embedding(tokens, t["e"], t["x"], scale=0.5, stream=stream),
                     lambda: cl.layernorm(t["x"], w, b, t["y"], residual=t["h"], h=t["h"], mean=t["mean"], rstd=t["rstd"], stream=stream),
                     lambda: cl.linear(t["y"], head, t["z"], transB=True, stream=stream),
                     lambda: cl.token_logprobs(t["z"], tokens, t["logp"], lse=t["lse"], entropy=t["H"], top_index=t["ti"], stream=stream),
                     lambda: cl.token_logprobs_backward(t["z"], tokens, t["lse"], t["dz"], dlogp=t["logp"], dentropy=dloss, entropy=t["H"], stream=stream)]
            if i:
                calls[3:] = [lambda: cl.distill(t["z"], index, values, t["loss"], lse=t["lse"], stream=stream),
                             lambda: cl.distill_backward(t["z"], index, values, t["lse"], dloss, t["z"], stream=stream),
                             lambda: cl.linear(t["z"], head, t["dy"], stream=stream)]
            else:
                calls.append(lambda: cl.linear(t["dz"], head, t["dy"], stream=stream))
            calls += [lambda: cl.layernorm_backward(t["dy"], t["h"], w, t["mean"], t["rstd"], t["dh"], t["dw"], t["db"], workspace=spaces[1], stream=stream),
                      lambda: cl.embedding_backward(t["dh"], tokens, t["dt"], workspace=spaces[0], accumulate=i == 1, stream=stream),
                      lambda: cl.embedding_backward(t["dy"], tokens, t["e"], scale=-0.1, workspace=spaces[0], accumulate=True, stream=stream)]
            for call in calls:
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
    assert cl.linear_status() == 0
    for k, v in slow.items():
        assert torch.isfinite(v.float()).all(), k
        assert torch.equal(v, fast[k]), k
        assert torch.equal(v, replayed[k]), k


def test_workspaces_of_calls_on_another_stream_are_not_memory_in_use(cl):
    """A block of the workspace's size is freed on the current stream while work that reads and writes it is still queued there; calls on
    another stream that bring no workspace compute as ever, and so does the queued work."""
    rng = np.random.default_rng(60)
    rows, cols, vocab = 600, 1024, 900
    h, dy = _rand(rng, (rows, cols), torch.float32), _rand(rng, (rows, cols), torch.float32)
    tokens = torch.tensor(_spread_tokens(rng, rows, vocab, "ranks"), device=_dev())
    mean = h.mean(1)
    rstd = torch.rsqrt((h - mean[:, None]).square().mean(1) + 1e-5)
    dx, dw, db, dt = torch.empty_like(h), torch.zeros(cols, device=_dev()), torch.zeros(cols, device=_dev()), torch.zeros(vocab, cols, device=_dev())
    cl.layernorm_backward(dy, h, None, mean, rstd, dx, dw, db)
    cl.embedding_backward(dy, tokens, dt)
    want_dw, want_dt = dw.clone(), dt.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=_dev())
    for size, call, got, want in (
            (cl.layernorm_backward_workspace(rows, cols), lambda s: cl.layernorm_backward(dy, h, None, mean, rstd, dx, dw, db, stream=s), dw, want_dw),
            (cl.embedding_backward_workspace(rows, vocab, cols), lambda s: cl.embedding_backward(dy, tokens, dt, stream=s), dt, want_dt)):
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


@pytest.mark.parametrize("rows,cols", [(1, 64), (5, 200), (40, 1001), (9, 4104), (300, 776), (3, 9000), (2, 17000)])
@pytest.mark.parametrize("h_t,dy_t", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_layernorm_of_operands_that_begin_differently(cl, rows, cols, h_t, dy_t):
    """Rows that lie differently in each operand leave the same values as rows that lie alike, and these the oracle's."""
    rng = np.random.default_rng(rows * 3 + cols)
    x, r = _rand(rng, (rows, cols), DT[dy_t]), _rand(rng, (rows, cols), DT[h_t])
    w, b = _rand(rng, cols + 3, torch.float32, 0.2) + 1, _rand(rng, cols + 3, torch.float32)
    one = lambda: torch.empty(rows, device=_dev())  # noqa: E731
    for wt, bt in ((w[:cols], b[:cols]), (w[1:cols + 1], b[3:])):
        h64, y64, _, r64 = ref.layernorm(_f64(x), _f64(r), _f64(wt), _f64(bt), float(np.float32(1e-5)))
        tol = _layernorm_tolerance(h64, _f64(wt), y64, r64, True)
        for pads in ((0, 0, 0, 0), (1, 2, 3, 5), (7, 0, 7, 0), (8, 16, 8, 0)):
            y, whole = _room(rows, cols, torch.float32, pads[2], pads[0] % 3)
            h, _ = _room(rows, cols, DT[h_t], pads[3], pads[1] % 2)
            mean, rstd = one(), one()
            cl.layernorm(_lay(x, pads[0], pads[3]), wt, bt, y, residual=_lay(r, pads[1], pads[2]), h=h, mean=mean, rstd=rstd)
            _close(y, y64, tol, "y")
            _close(h, h64, U * np.abs(h64), "h")
            _untouched(whole, cols)
            dx, whole = _room(rows, cols, DT[h_t], pads[1], pads[2] % 3)
            dw, db = torch.empty(cols, device=_dev()), torch.empty(cols, device=_dev())
            cl.layernorm_backward(_lay(x, pads[3], pads[0]), h, wt, mean, rstd, dx, dw, db, dres=_lay(r, pads[0], pads[1]))
            h_, dy_, m_, s_, w_ = _f64(h), _f64(x), _f64(mean), _f64(rstd), _f64(wt)
            dx64, dw64, db64 = ref.layernorm_backward(dy_, h_, w_, m_, s_, _f64(r))
            # (as in test_layernorm_backward)
            xh, q = np.abs(h_ - m_[:, None]) * s_[:, None], np.abs(dy_ * w_)
            qx, q1 = (q * xh).mean(axis=1, keepdims=True), q.mean(axis=1, keepdims=True)
            dtol = s_[:, None] * (4 * U * q + (SUM + 4 * U) * q1 + xh * (SUM + 15 * U) * qx) + 2 * U * np.abs(_f64(r)) + 2 * U * np.abs(dx64)
            _close(dx, dx64, dtol, "dx")
            _untouched(whole, cols)
            _close(dw, dw64, (SUM + 4 * U) * (np.abs(dy_) * xh).sum(axis=0), "dw")
            _close(db, db64, SUM * np.abs(dy_).sum(axis=0), "db")


def test_layernorm_backward_shares_of_rows_that_begin_differently(cl):
    """Integers, exact in any order: many rows of lengths whose rows begin at every place of a line, and none lost at their ends."""
    rng = np.random.default_rng(77)
    for rows, cols in ((700, 65), (3000, 67), (900, 769), (640, 1029), (800, 2051), (500, 4097), (330, 5123), (310, 8195)):
        dy, h = (_put(rng.integers(-4, 5, size=(rows, cols)), torch.bfloat16) for _ in range(2))
        one, zero = torch.ones(rows, device=_dev()), torch.zeros(rows, device=_dev())
        dx, dw, db = torch.empty_like(h), torch.full((cols + 1,), 7.0, device=_dev()), torch.full((cols + 1,), 7.0, device=_dev())
        cl.layernorm_backward(dy, h, None, zero, one, dx, dw[:cols], db[:cols])
        assert torch.equal(dw[:cols], (dy.float() * h.float()).sum(0)) and torch.equal(db[:cols], dy.float().sum(0)), (rows, cols)
        assert float(dw[cols]) == 7.0 and float(db[cols]) == 7.0


def test_scores_beyond_32_bits_of_offset(cl):
    """A matrix of more than 2^31 elements: its last rows leave what the same rows leave by themselves."""
    rows, vocab, few = 17000, 131072, 5
    gen = torch.Generator(device=_dev()).manual_seed(1)
    x = torch.empty(rows, vocab, dtype=torch.bfloat16, device=_dev())
    for at in range(0, rows, 1000):
        x[at:at + 1000] = torch.randn(min(1000, rows - at), vocab, generator=gen, device=_dev())
    t = torch.randint(0, vocab, (rows,), generator=gen, device=_dev())
    one = lambda n: torch.full((n,), float("nan"), device=_dev())  # noqa: E731
    logp, lse, h, ti = one(rows), one(rows), one(rows), torch.empty(rows, 5, dtype=torch.int32, device=_dev())
    cl.token_logprobs(x, t, logp, lse=lse, entropy=h, top_index=ti)
    assert torch.isfinite(logp).all() and torch.isfinite(lse).all() and torch.isfinite(h).all()
    up = torch.full((rows,), -1.0, device=_dev())
    tail, part = x[-few:].clone(), slice(rows - few, rows)
    logp2, lse2, h2, ti2 = one(few), one(few), one(few), torch.empty(few, 5, dtype=torch.int32, device=_dev())
    cl.token_logprobs(tail, t[part], logp2, lse=lse2, entropy=h2, top_index=ti2)
    # (another number of CTAs a row: other sums of the same terms, 64 U of each)
    for a, b in ((logp[part], logp2), (lse[part], lse2), (h[part], h2)):
        assert torch.allclose(a, b, rtol=2 * SUM, atol=2 * SUM)
    assert torch.equal(ti[part], ti2)
    index, values = torch.randint(0, vocab, (rows, 6), generator=gen, device=_dev()), torch.randn(rows, 6, generator=gen, device=_dev())
    loss, loss2 = one(rows), one(few)
    cl.distill(x, index, values, loss)
    cl.distill(tail, index[part], values[part], loss2)
    assert torch.isfinite(loss).all() and torch.allclose(loss[part], loss2, rtol=2 * SUM, atol=16 * SUM)
    want = torch.empty_like(tail)
    cl.token_logprobs_backward(tail, t[part], lse[part], want, dlogp=up[part])
    cl.token_logprobs_backward(x, t, lse, x, dlogp=up)
    assert torch.equal(_bits(x[part]), _bits(want)) and torch.isfinite(x[::1000].float()).all()


def test_rows_beyond_32_bits_of_offset(cl):
    """Layer norm, lookup and gradient over more than 2^31 elements: their last rows are right, and so are whole sums of integers."""
    rows, cols = 530000, 4104
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device=_dev())
    x[:, ::2] = 3.0                                                         # mean 2, variance 1
    x[-1, :] = torch.arange(cols, device=_dev()) % 7
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=_dev()), torch.empty(rows, device=_dev())
    cl.layernorm(x, None, None, y, mean=mean, rstd=rstd, eps=0.0)
    assert torch.all(mean[:-1] == 2) and torch.all((rstd[:-1] - 1).abs() <= 2 * U) and torch.all(y[-3:-1, ::2] == 1) and torch.all(y[-3:-1, 1::2] == -1)
    last = x[-1].double()
    assert abs(float(mean[-1] - last.mean())) < 1e-5
    dw, db, one, zero = torch.empty(cols, device=_dev()), torch.empty(cols, device=_dev()), torch.ones(rows, device=_dev()), torch.zeros(rows, device=_dev())
    x[-1] = 1.0
    cl.layernorm_backward(x, x, None, zero, one, y, dw, db)                 # dy = h: dw the sum of squares
    assert torch.equal(db[1::2], torch.full_like(db[1::2], rows)) and torch.equal(db[::2], torch.full_like(db[::2], 3 * rows - 2))
    assert torch.equal(dw[::2], torch.full_like(dw[::2], 9 * rows - 8))
    tokens = torch.arange(rows, device=_dev()) % 3
    tokens[-1] = 5
    dt = torch.empty(8, cols, device=_dev())
    cl.embedding_backward(x, tokens, dt)
    count = torch.bincount(tokens, minlength=8).float()
    assert torch.equal(dt[:, 1], count) and torch.equal(dt[5], torch.ones(cols, device=_dev()))
    assert torch.equal(dt[:3, 0], 3 * count[:3])
    cl.embedding(tokens, dt[:, :].to(torch.bfloat16), y)
    assert torch.all(y[-1] == 1) and torch.equal(y[-2, :2].float(), dt[int(tokens[-2]), :2].to(torch.bfloat16).float())


@pytest.mark.parametrize("k", [2, 7, 32, 40, 100, 256])
@pytest.mark.parametrize("x_t,t_t", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("normalize", [True, False])
def test_distill_of_a_teacher_with_nan_and_infinities(cl, k, x_t, t_t, normalize):
    """A NaN or +infinity among a row's values beside empty entries and behind the last one: they stay no places, the row's results are
    what the formula gives, and other rows' are as without it."""
    rng = np.random.default_rng(k)
    rows, vocab, scale = 12, 700, 1.5
    x = _rand(rng, (rows, vocab), DT[x_t], 2.0)
    index, values = rng.integers(0, vocab, size=(rows, k)), rng.normal(size=(rows, k))
    index[:, 1::3] = -1
    index[3, 1] = vocab
    plain = torch.tensor(values, dtype=torch.float32).to(DT[t_t]).to(_dev())
    values[1, 0] = float("nan")
    values[3, 0] = INF
    values[4, 0] = 3e38                                                     # infinite once it is scaled
    values[6, 1] = float("nan")                                             # in an empty entry: it does not matter
    values[7, 0], values[7, k - 1] = -INF, float("nan")
    index[8] = -1                                                           # nothing but empty entries
    values[8] = float("nan")
    it, vt = torch.tensor(index, device=_dev()), torch.tensor(values, dtype=torch.float32).to(DT[t_t]).to(_dev())
    dloss = _rand(rng, rows, torch.float32)
    dloss[3] = 0.0
    f = lambda: torch.full((rows,), 7.0, device=_dev())  # noqa: E731
    got = [f(), f(), torch.full_like(x, 7.0)]
    ref_ = [f(), f(), torch.full_like(x, 7.0)]
    for (loss, lse, dx), v in ((got, vt), (ref_, plain)):
        cl.distill(x, it, v, loss, lse=lse, scale=scale, normalize=normalize)
        cl.distill_backward(x, it, v, lse, dloss, dx, scale=scale, normalize=normalize)
    v64 = _f64(vt)
    v64[4, 0] = INF                                                         # (1.5 times 3e38 is, in fp32)
    with np.errstate(all="ignore"):
        want, _, _ = ref.distill(_f64(x), index, v64, scale, normalize)
        want_dx, _ = ref.distill_backward(_f64(x), index, v64, _f64(got[1]), _f64(dloss), scale, normalize)
    loss, dx = _f64(got[0]), _f64(got[2])
    broken = [r for r in range(rows) if not np.isfinite(want[r])]
    assert broken == ([1, 3, 4] if index[7, k - 1] < 0 else [1, 3, 4, 7])
    assert np.array_equal(loss[broken], want[broken], equal_nan=True)
    assert not np.isfinite(dx[[r for r in broken if r != 3]]).any() and not np.isfinite(want_dx[[r for r in broken if r != 3]]).any()
    assert not dx[3].any() and not dx[8].any() and loss[8] == 0
    assert torch.equal(_bits(got[1]), _bits(ref_[1]))
    same = [r for r in range(rows) if r not in (1, 3, 4, 7, 8)]
    assert torch.equal(_bits(got[0][same]), _bits(ref_[0][same])) and torch.equal(_bits(got[2][same]), _bits(ref_[2][same]))


@pytest.mark.parametrize("shift", [0.0, 300.0, 3000.0, 30000.0, -30000.0])
@pytest.mark.parametrize("vocab", [700, 50257])
@pytest.mark.parametrize("x_t,scale", [("f32", 0.7), ("bf16", 1.0)])
def test_log_probabilities_of_rows_far_from_zero(cl, shift, vocab, x_t, scale):
    """log p = scale (x - largest) - log(sum): its error is that of these two, however large the scores are; never above 0.  A term e^d
    is off by (4 + 3 |d|) U, their sum by 64 U more; the logarithm by 4 U, the difference and the last sum by U each."""
    rng = np.random.default_rng(vocab)
    rows, top, s = 20, 8, float(np.float32(scale))
    x = rng.normal(size=(rows, vocab)) * 3 + shift
    x[:6, 5] = shift + 40.0                                                 # sure of one place
    x[6:9] = shift
    x[9, 3] = -INF
    x = torch.tensor(x, dtype=torch.float32).to(DT[x_t]).to(_dev())
    x64 = _f64(x)
    tokens = rng.integers(0, vocab, size=rows)
    tokens[:3], tokens[9] = 5, 3
    tokens[10:] = x64[10:].argmax(axis=1)
    w_logp, w_lse, _, w_tv, w_ti = ref.logprobs(x64, tokens, s, top)
    ed, _, _ = _row_spread(x64, s)
    rest = w_lse - s * x64.max(axis=1)
    sums = SUM + (4 + 3 * ed) * U + 4 * U * np.abs(rest)
    far = lambda at: np.where(np.isfinite(at), np.abs(s * (at - x64.max(axis=1, keepdims=True))), 0.0)  # noqa: E731
    f = lambda: torch.full((rows,), float("nan"), device=_dev())  # noqa: E731
    logp, lse, tv = f(), f(), torch.empty(rows, top, device=_dev())
    cl.token_logprobs(x, torch.tensor(tokens, device=_dev()), logp, lse=lse, top_values=tv, scale=scale)
    _close(logp, w_logp, sums + 2 * U * far(np.take_along_axis(x64, tokens[:, None], 1))[:, 0], "logp")
    _close(tv, w_tv, sums[:, None] + 2 * U * far(np.take_along_axis(x64, w_ti, 1)), "top values")
    assert (logp <= 0).all() and (tv <= 0).all()
    alone = f()
    cl.token_logprobs(x, torch.tensor(tokens, device=_dev()), alone, scale=scale)
    assert torch.allclose(alone, logp, rtol=2 * SUM, atol=2 * SUM)          # (another number of CTAs a row)
    # a teacher that is as sure: the loss is a difference of logarithms as small as these
    values = _put(rng.normal(size=(rows, top)), torch.float32)
    loss = f()
    cl.distill(x, torch.tensor(w_ti, device=_dev()), values, loss, scale=scale)
    w_loss, _, size = ref.distill(x64, w_ti, _f64(values), s, True)
    spread = np.abs(s * _f64(values)).max(axis=1)
    q_err = SUM + (4 + 6 * spread) * U
    _close(loss, w_loss, size * (q_err + 4 * U) + sums + q_err + 2 * U * far(np.take_along_axis(x64, w_ti, 1)).max(axis=1), "loss")


@pytest.mark.parametrize("cols", [41, 47, 61, 328, 440, 776, 856, 1001, 2568, 4112, 5120, 9224, 16376, 20560])
@pytest.mark.parametrize("x_t", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 3])
def test_layernorm_of_constant_rows_of_any_length(cl, cols, x_t, pad):
    """The sum of a row of ones is exact and so is its mean, whether or not the length has an exact reciprocal: y is the bias, however
    small eps is.  A constant dy has no gradient where the normalised values have mean 0."""
    rng = np.random.default_rng(cols)
    b = _rand(rng, cols, torch.float32)
    half, one = torch.full((5, cols), 0.5, device=_dev()), torch.ones(5, cols, dtype=DT[x_t], device=_dev())
    mean, rstd, scale = (torch.empty(5, device=_dev()) for _ in range(3))
    for eps in (1e-5, 1e-12):
        for x, r in ((one, None), (half.to(DT[x_t]), half)):
            y, _ = _room(5, cols, torch.float32, pad)
            cl.layernorm(x, None, b, y, residual=r, mean=mean, rstd=rstd, eps=eps)
            assert torch.all(mean == 1) and torch.equal(y, b.expand(5, -1))
            assert torch.all((rstd * eps ** 0.5 - 1).abs() < 1e-6)
        code = torch.empty(5, cols, dtype=torch.float8_e4m3fn, device=_dev())
        cl.layernorm(one, None, None, code, scale=scale, eps=eps)
        assert not scale.any() and not code.float().any()
    h = torch.ones(5, cols, device=_dev())
    h[:, 1::2] = -1.0
    h[:, -1] = 0.0 if cols % 2 else -1.0
    dx, _ = _room(5, cols, torch.float32, pad)
    cl.layernorm_backward(one, h, None, torch.zeros(5, device=_dev()), torch.full((5,), 1e6, device=_dev()), dx)
    assert not dx.any()


@pytest.mark.parametrize("cols", [40, 264, 1000, 1032, 2600, 5120, 9000, 20000])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("size", [2.0 ** -66, 2.0 ** -40])
def test_layernorm_of_very_small_rows(cl, cols, pad, size):
    """With eps = 0 the normalised values do not know the rows' size: y of size h is that of h to the bit (size a power of two), and dx that of
    h, over the size.  (Squares of 2^-66 are 2^-132: what of them is lost below 2^-149 is 2^-17 of one at most, and 64 U of their sum.)"""
    rng = np.random.default_rng(cols)
    h = _lay(_rand(rng, (9, cols), torch.float32), pad)
    hs = _lay(h * size, pad)
    dy, w = _lay(100 * _rand(rng, (9, cols), torch.float32), pad), _rand(rng, cols, torch.float32, 0.2) + 1
    out = []
    for x in (h, hs):
        y, mean, rstd = _lay(torch.empty_like(h), pad), torch.empty(9, device=_dev()), torch.empty(9, device=_dev())
        cl.layernorm(x, None, None, y, mean=mean, rstd=rstd, eps=0.0)
        dx, dw, db = _lay(torch.empty_like(h), pad), torch.empty(cols, device=_dev()), torch.empty(cols, device=_dev())
        out.append((y, mean, rstd, dx, dw, db))
    y, mean, rstd, _, _, _ = out[0]
    y2, mean2, rstd2, _, _, _ = out[1]
    lost = 2.0 ** -17
    assert torch.equal(mean2, mean * size) and ((rstd2.double() * size / rstd - 1).abs() <= lost + SUM).all()
    assert ((y2 - y).abs() <= (lost + SUM) * y.abs()).all()
    for x, m, r, (_, _, _, dx, dw, db) in ((h, mean, rstd, out[0]), (hs, mean * size, rstd / size, out[1])):
        cl.layernorm_backward(dy, x, w, m, r, dx, dw, db)
    (_, _, _, dx, dw, db), (_, _, _, dx2, dw2, db2) = out
    assert torch.isfinite(dx).all() and torch.isfinite(dx2).all()
    assert torch.equal(db2, db) and torch.equal(dw2, dw) and torch.equal(dx2 * size, dx)


@pytest.mark.parametrize("n,vocab,cols", [(1, 9, 1), (40, 17, 264), (900, 500, 33), (4097, 300, 72), (30000, 3, 24), (2000, 20000, 7)])
@pytest.mark.parametrize("dy_t,ids,pad,shift", [("bf16", "i32", 3, 1), ("f32", "i64", 5, 3), ("bf16", "i64", 1, 0), ("f32", "i32", 0, 7)])
def test_embedding_backward_into_a_bf16_table_with_a_pitch(cl, n, vocab, cols, dy_t, ids, pad, shift):
    """Integers: their sums are exact in fp32 in any order, and each row is rounded to bf16 once; what lies between the rows and before
    the table stays."""
    rng = np.random.default_rng(n + cols)
    tokens = _spread_tokens(rng, n, vocab, "ranks")
    dy = _lay(_put(rng.integers(-8, 9, size=(n, cols)), DT[dy_t]), pad, shift)
    t = torch.tensor(tokens, dtype=DT[ids], device=_dev())
    ok = (t >= 0) & (t < vocab)
    want = torch.zeros(vocab, cols, dtype=torch.float64, device=_dev()).index_add_(0, t[ok].long(), dy[ok].double()).float()
    before = _put(rng.integers(-8, 9, size=(vocab, cols)), torch.bfloat16)
    store = torch.full((shift + vocab * (cols + pad),), 7.0, dtype=torch.bfloat16, device=_dev())
    whole = store[shift:].view(vocab, cols + pad)
    dt = whole[:, :cols]
    for accumulate, result in ((False, want.bfloat16()), (True, (before.float() + 2 * want).bfloat16())):
        dt.copy_(before)
        cl.embedding_backward(dy, t, dt, scale=2.0 if accumulate else 1.0, accumulate=accumulate)
        assert torch.equal(dt, result)
        _untouched(whole, cols)
        assert torch.all(store[:shift] == 7.0)


@pytest.mark.parametrize("x_t", ["bf16", "f32"])
def test_scores_of_more_rows_than_a_grid_has(cl, x_t):
    """65535 rows are a grid's second dimension, what is above goes to the third: rows on both sides, the last one and the first are as
    by themselves, all of them right, and nothing behind them is written."""
    rows, vocab, k, behind = 65535 + 7, 41, 5, 3
    gen = torch.Generator(device=_dev()).manual_seed(2)
    x = torch.randn(rows, vocab, generator=gen, device=_dev()).mul_(2).to(DT[x_t])
    t = torch.randint(-1, vocab, (rows,), generator=gen, device=_dev())
    index, values = torch.randint(-1, vocab, (rows, k), generator=gen, device=_dev()), torch.randn(rows, k, generator=gen, device=_dev())
    up = torch.randn(rows, generator=gen, device=_dev())

    def outputs(a, b):
        n = b - a
        f = lambda *s, d=torch.float32: torch.full((n + behind, *s), 7, dtype=d, device=_dev())  # noqa: E731
        out = dict(logp=f(), lse=f(), H=f(), lse2=f(), tv=f(k), ti=f(k, d=torch.int32), dx=f(vocab, d=DT[x_t]), loss=f(), lse3=f(), dx2=f(vocab, d=DT[x_t]))
        o = {q: v[:n] for q, v in out.items()}
        cl.token_logprobs(x[a:b], t[a:b], o["logp"], lse=o["lse"], entropy=o["H"])
        cl.token_logprobs(x[a:b], lse=o["lse2"], top_values=o["tv"], top_index=o["ti"])
        cl.token_logprobs_backward(x[a:b], t[a:b], o["lse"], o["dx"], dlogp=up[a:b], dentropy=up[a:b], entropy=o["H"])
        cl.distill(x[a:b], index[a:b], values[a:b], o["loss"], lse=o["lse3"])
        cl.distill_backward(x[a:b], index[a:b], values[a:b], o["lse"], up[a:b], o["dx2"])
        assert all(torch.all(v[n:] == 7) for v in out.values())
        return o

    whole = outputs(0, rows)
    for a, b in ((0, 9), (65530, 65536), (65536, rows), (rows - 1, rows)):
        for q, v in outputs(a, b).items():
            assert torch.equal(_bits(whole[q][a:b]), _bits(v)), (q, a)
    lp = torch.log_softmax(x.double(), 1)
    assert torch.allclose(whole["lse"].double(), torch.logsumexp(x.double(), 1), rtol=SUM, atol=SUM)
    assert torch.allclose(whole["logp"].double(), torch.where(t >= 0, lp.gather(1, t.clamp_min(0)[:, None])[:, 0], 0.0), rtol=SUM, atol=SUM)
    assert torch.equal(whole["ti"].long(), x.double().sort(dim=1, descending=True, stable=True).indices[:, :k])


@pytest.mark.parametrize("vocab,k", [(300, 64), (50257, 20), (4097, 1)])
@pytest.mark.parametrize("x_t", ["bf16", "f32"])
def test_top_places_are_a_teacher(cl, vocab, k, x_t):
    """A teacher's best places and their log probabilities, as token_logprobs leaves them, teach a student without normalizing; the teacher
    itself has nothing left to learn: its loss is 0 and its gradient what the places that are not among the best have of the sum."""
    rng = np.random.default_rng(vocab + k)
    rows = 24
    teacher, student = _scores(rng, rows, vocab, x_t, False), _scores(rng, rows, vocab, x_t, False)
    student[:, torch.isinf(teacher[0])] = -INF
    student[:, ~torch.isinf(teacher[0])] = student[:, ~torch.isinf(teacher[0])].clamp_min(-9.0)      # a place that the teacher names is not masked
    tv, ti = torch.empty(rows, k, device=_dev()), torch.empty(rows, k, dtype=torch.int32, device=_dev())
    f = lambda: torch.full((rows,), float("nan"), device=_dev())  # noqa: E731
    cl.token_logprobs(teacher, top_values=tv, top_index=ti)
    dloss = _rand(rng, rows, torch.float32)
    at, v64 = ti.cpu().numpy().astype(np.int64), _f64(tv)
    for x in (student, teacher):
        loss, lse, dx = f(), f(), torch.empty(rows, vocab, device=_dev())
        cl.distill(x, ti, tv, loss, lse=lse, normalize=False)
        cl.distill_backward(x, ti, tv, lse, dloss, dx, normalize=False)
        x64 = _f64(x)
        w_loss, _, size = ref.distill(x64, at, v64, 1.0, False)
        lse_tol, _ = _statistics_tolerance(x64, 1.0)
        q_err = SUM + (4 + 6 * np.abs(v64).max(axis=1)) * U                 # (as in test_distill)
        biggest = np.array([np.abs(r[np.isfinite(r)]).max() for r in x64])
        _close(loss, w_loss, size * (q_err + 4 * U) + lse_tol + q_err + 4 * U * biggest, "loss")
        want, terms = ref.distill_backward(x64, at, v64, _f64(lse), _f64(dloss), 1.0, False)
        far = np.where(np.isfinite(x64), np.abs(x64 - _f64(lse)[:, None]), 0.0)
        _close(dx, want, terms * ((3 * far + 16) * U + q_err[:, None]) + 1e-37, "dx")
    # (the teacher against itself: each term is the difference of two equal logarithms)
    assert (np.abs(w_loss) <= 2 * U * (np.abs(v64).max(axis=1) + 1)).all()
    named = torch.zeros(rows, vocab, dtype=torch.bool, device=_dev()).scatter_(1, ti.long(), True)
    assert torch.all((dx * dloss[:, None])[~named] >= 0)
