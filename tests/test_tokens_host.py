"""Host side of the operators on tokens and of layer norm, no GPU: struct layouts, workspace sizes, and the refusals, which come
before anything touches a device (the addresses below are never dereferenced)."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVAL, UNSUPPORTED, CUDA = -1, -2, -6
BIG = 1 << 33


@pytest.fixture(scope="module")
def ops():
    import paper_2512_22142_b200 as cl
    return cl.ops


def test_struct_layouts_match_the_header(ops, tmp_path):
    names = {"embedding": ops._Embedding, "embedding_backward": ops._EmbeddingBackward, "layernorm": ops._Layernorm, "layernorm_backward": ops._LayernormBackward,
             "logprobs": ops._Logprobs, "logprobs_backward": ops._LogprobsBackward, "distill": ops._Distill, "distill_backward": ops._DistillBackward}
    lines = []
    for name, cls in names.items():
        lines.append(f'printf("%zu\\n", sizeof(cleave_{name}_t));')
        lines += [f'printf("%zu\\n", offsetof(cleave_{name}_t, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "cleave.h"\nint main(void) {' + "".join(lines) + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for cls in names.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f[0]).offset for f in cls._fields_]
    assert got == want


def _call(ops, name, cls, base, kw, ws=()):
    d = cls()
    for k, v in {**base, **kw}.items():
        setattr(d.f if hasattr(d, "f") and hasattr(d.f, k) else d, k, v)
    return getattr(ops.lib, name)(ctypes.byref(d), *ws, None)


def _embedding(ops, **kw):
    return _call(ops, "cleave_embedding", ops._Embedding, dict(n=4, vocab=10, cols=8, id_type=4, table_type=1, out_type=2, scale=1.0, ids=4096, table=8192, ldt=8, out=16384, ldo=8), kw)


def _embedding_bwd(ops, ws=4096, **kw):
    return _call(ops, "cleave_embedding_backward", ops._EmbeddingBackward,
                 dict(n=4, vocab=10, cols=8, id_type=5, dy_type=1, dtable_type=2, scale=1.0, ids=4096, dy=8192, lddy=8, dtable=16384, lddt=8), kw, (ws,))


def _layernorm(ops, **kw):
    return _call(ops, "cleave_layernorm", ops._Layernorm, dict(rows=4, cols=8, eps=1e-5, x_type=1, x=4096, ldx=8, y_type=1, y=8192, ldy=8), kw)


def _layernorm_bwd(ops, ws=4096, **kw):
    return _call(ops, "cleave_layernorm_backward", ops._LayernormBackward,
                 dict(rows=4, cols=8, dy_type=1, dy=4096, lddy=8, h_type=1, h=8192, ldh=8, mean=4096, rstd=4096, dx=16384, lddx=8, dw=4096, db=4096), kw, (ws,))


def _logprobs(ops, **kw):
    return _call(ops, "cleave_logprobs", ops._Logprobs, dict(rows=4, cols=100, x_type=1, id_type=4, top=3, scale=1.0, x=4096, ldx=100, ids=4096, logp=8192, lse=8192,
                                                             entropy=8192, top_values=8192, ldtv=3, top_index=8192, ldti=3), kw)


def _logprobs_bwd(ops, **kw):
    return _call(ops, "cleave_logprobs_backward", ops._LogprobsBackward, dict(rows=4, cols=100, x_type=1, id_type=5, dx_type=2, scale=1.0, x=4096, ldx=100, ids=4096, lse=8192,
                                                                              entropy=8192, dlogp=8192, dlse=8192, dentropy=8192, dx=16384, lddx=100), kw)


DISTILL = dict(rows=4, cols=100, k=5, x_type=1, index_type=4, values_type=2, normalize=1, scale=1.0, x=4096, ldx=100, index=4096, ldindex=5, values=8192, ldvalues=5, loss=8192, lse=8192)


def _distill(ops, **kw):
    return _call(ops, "cleave_distill", ops._Distill, DISTILL, kw)


def _distill_bwd(ops, **kw):
    return _call(ops, "cleave_distill_backward", ops._DistillBackward, dict(DISTILL, loss=None, dloss=4096, dx_type=1, dx=16384, lddx=100), kw)


NAN, INF = float("nan"), float("inf")
REFUSED = [
    (_embedding, [dict(cols=0), dict(vocab=0), dict(ids=None), dict(id_type=1), dict(id_type=0), dict(ids=4098), dict(id_type=5, ids=4100), dict(table=None), dict(table_type=3),
                  dict(table=8193), dict(ldt=7), dict(out=None), dict(out_type=0), dict(out=16386), dict(ldo=4), dict(scale=NAN), dict(scale=INF), dict(ldo=1 << 41)]),
    (_embedding_bwd, [dict(cols=0), dict(vocab=0), dict(ids=None), dict(id_type=3), dict(ids=4100), dict(dy=None), dict(dy_type=3), dict(lddy=7), dict(dtable=None),
                      dict(dtable_type=3), dict(dtable=16386), dict(lddt=7), dict(accumulate=2), dict(scale=-INF), dict(ws=None), dict(ws=4100), dict(n=0, ws=None), dict(n=0, dtable=None)]),
    (_layernorm, [dict(cols=0), dict(x=None), dict(x_type=0), dict(x_type=3), dict(ldx=7), dict(x=4097), dict(y_type=3), dict(scale=4096), dict(y_type=3, scale=4097),
                  dict(h=4096, ldh=8), dict(r=4096), dict(r_type=1, r=4096, ldr=4), dict(r_type=2, r=4098, ldr=8), dict(w=4096), dict(w_type=3, w=4096), dict(b=4096),
                  dict(b_type=2, b=4098), dict(mean=4098), dict(rstd=4098), dict(eps=-1.0), dict(eps=NAN), dict(y=None), dict(ldy=1 << 41),
                  dict(r_type=1, r=4096, ldr=8, h=4097, ldh=8)]),
    (_layernorm_bwd, [dict(cols=0), dict(dy=None), dict(dy_type=3), dict(lddy=4), dict(h_type=0), dict(h=8193), dict(dx=None), dict(lddx=7), dict(mean=None), dict(mean=4098),
                      dict(rstd=None), dict(rstd=4098), dict(ws=None), dict(ws=4100), dict(dres=4097, lddres=8), dict(dres=4096, lddres=2), dict(dw=4098), dict(db=4098),
                      dict(w=4096), dict(db=None, ws=None), dict(dw=None, ws=None)]),
    (_logprobs, [dict(cols=0), dict(x=None), dict(x_type=3), dict(x=4097), dict(ldx=99), dict(ids=None), dict(id_type=0), dict(id_type=2), dict(id_type=5, ids=4100), dict(top=0),
                 dict(top=3, top_values=None, top_index=None), dict(cols=2, top=3), dict(ldtv=2), dict(ldti=2), dict(top_values=8194), dict(top_index=8193), dict(logp=8194),
                 dict(lse=8193), dict(entropy=8194), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(logp=None),
                 dict(logp=None, ids=None, id_type=0, lse=None, entropy=None, top=0, top_values=None, top_index=None)]),
    (_logprobs_bwd, [dict(cols=0), dict(x=None), dict(x_type=3), dict(ldx=99), dict(ids=None), dict(ids=4100), dict(lse=None), dict(lse=4098), dict(entropy=None), dict(dentropy=None),
                     dict(dlogp=4098), dict(dlse=4097), dict(dentropy=4098), dict(dx=None), dict(dx_type=3), dict(dx=16386), dict(lddx=99), dict(scale=0.0), dict(scale=NAN),
                     dict(dlogp=None), dict(dlogp=None, ids=None, id_type=0, dlse=None, dentropy=None, entropy=None)]),
    (_distill, [dict(cols=0), dict(k=0), dict(x=None), dict(x_type=3), dict(ldx=99), dict(index=None), dict(index_type=2), dict(index=4098), dict(ldindex=4), dict(values=None),
                dict(values_type=3), dict(values=8194), dict(ldvalues=4), dict(normalize=2), dict(scale=0.0), dict(scale=INF), dict(loss=None), dict(loss=4098), dict(lse=4098)]),
    (_distill_bwd, [dict(cols=0), dict(k=0), dict(x=None), dict(ldx=99), dict(index=None), dict(values=None), dict(lse=None), dict(lse=4098), dict(dloss=None), dict(dloss=4098),
                    dict(dx=None), dict(dx_type=0), dict(dx=16385), dict(lddx=99), dict(scale=-2.0)]),
]


@pytest.mark.parametrize("call,kw", [(c, kw) for c, many in REFUSED for kw in many])
def test_refused(ops, call, kw):
    assert call(ops, **kw) == INVAL


@pytest.mark.parametrize("call,kw", [(_embedding, dict(n=1 << 31)), (_embedding, dict(vocab=1 << 31)), (_embedding, dict(cols=1 << 31, ldt=BIG, ldo=BIG)),
                                     (_embedding_bwd, dict(n=1 << 31)), (_embedding_bwd, dict(vocab=(1 << 32) - 1)), (_embedding_bwd, dict(cols=1 << 31, lddy=BIG, lddt=BIG)),
                                     (_layernorm, dict(rows=1 << 31)), (_layernorm, dict(cols=1 << 31, ldx=BIG, ldy=BIG)), (_layernorm_bwd, dict(rows=1 << 31)),
                                     (_layernorm_bwd, dict(cols=(1 << 32) - 1, lddy=BIG, ldh=BIG, lddx=BIG)), (_logprobs, dict(rows=1 << 31)), (_logprobs, dict(cols=1 << 31, ldx=BIG)),
                                     (_logprobs, dict(top=65, ldtv=65, ldti=65)), (_logprobs_bwd, dict(rows=1 << 31)), (_logprobs_bwd, dict(cols=1 << 31, ldx=BIG, lddx=BIG)),
                                     (_distill, dict(k=257, ldindex=257, ldvalues=257)), (_distill, dict(rows=1 << 31)), (_distill_bwd, dict(k=1000, ldindex=1000, ldvalues=1000)),
                                     (_distill_bwd, dict(cols=1 << 31, ldx=BIG, lddx=BIG))])
def test_beyond_the_limits(ops, call, kw):
    assert call(ops, **kw) == UNSUPPORTED


def test_nothing_to_do_needs_no_buffers(ops):
    assert _embedding(ops, n=0, ids=None, table=None, out=None) == 0
    assert _layernorm(ops, rows=0, x=None, y=None) == 0
    assert _logprobs(ops, rows=0, x=None, ids=None) == 0
    assert _logprobs_bwd(ops, rows=0, x=None, dx=None) == 0
    assert _distill(ops, rows=0, x=None, loss=None) == 0 and _distill_bwd(ops, rows=0, x=None, dx=None) == 0
    for name in ("cleave_embedding", "cleave_layernorm", "cleave_logprobs", "cleave_logprobs_backward", "cleave_distill", "cleave_distill_backward"):
        assert getattr(ops.lib, name)(None, None) == INVAL
    assert ops.lib.cleave_embedding_backward(None, 4096, None) == INVAL and ops.lib.cleave_layernorm_backward(None, 4096, None) == INVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="what a machine without a GPU answers")
def test_without_a_device_the_calls_say_so(ops):
    for call in (_embedding, _embedding_bwd, _layernorm, _layernorm_bwd, _logprobs, _logprobs_bwd, _distill, _distill_bwd):
        assert call(ops) == CUDA


def test_workspaces(ops):
    assert ops.layernorm_backward_workspace(0, 100) == 0 and ops.layernorm_backward_workspace(1, 100) >= 800
    assert ops.layernorm_backward_workspace((1 << 31) - 1, 100) <= 2 * 100 * 4 * 4096          # bounded: partial sums, not rows
    fn = ops.embedding_backward_workspace
    assert fn(0, 1000, 64) >= 4 * 1001 and fn(100, 1000, 64) >= 4 * 1101
    for n in (1, 100, 10 ** 5, (1 << 31) - 1):
        assert fn(n, 1000, 64) % 4 == 0 and fn(n, 1000, 64) <= 8 * n + 4 * 1001 + 64 + (8 + 2 * 4 * 64) * min(n, 4096)      # places with their tokens, offsets, pieces


def test_binding_refuses_what_the_library_cannot_see(ops):
    x, w, t = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: ops.embedding(t, x, x), lambda: ops.embedding_backward(x, t, x), lambda: ops.layernorm(x, w, w, x), lambda: ops.layernorm(x[0], w, w, x),
                 lambda: ops.layernorm_backward(x, x, w, w, w, x), lambda: ops.token_logprobs(x, t, w), lambda: ops.token_logprobs_backward(x, t, w, x, dlogp=w),
                 lambda: ops.distill(x, t[None], x, w), lambda: ops.distill_backward(x, t[None], x, w, w, x)):
        with pytest.raises(ValueError):
            call()


def _at(device, *size, dtype=torch.float32):
    """A tensor without memory that says it is on a GPU: the refusals come before anything else."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        return torch.empty(*size, dtype=dtype, device=device)


def test_binding_refuses_shapes_and_types(ops):
    here = lambda *s, **k: _at("cuda:0", *s, **k)  # noqa: E731
    x, y, w, v, ids, half = here(6, 8), here(6, 8), here(8), here(6), here(6, dtype=torch.int64), here(6, dtype=torch.int16)
    table, code, iv = here(20, 8), here(6, 8, dtype=torch.float8_e4m3fn), here(6, 3, dtype=torch.int32)
    tv, at, wrong = here(6, 3), here(6, 5, dtype=torch.int64), here(6, 5)
    bad = [lambda: ops.embedding(half, table, x, stream=1), lambda: ops.embedding(ids[:5], table, x, stream=1), lambda: ops.embedding(None, table, x, stream=1),
           lambda: ops.embedding(ids, table, here(6, 9), stream=1), lambda: ops.embedding(ids, table, code, stream=1), lambda: ops.embedding(ids, here(20), x, stream=1),
           lambda: ops.embedding(here(12, dtype=torch.int64)[::2], table, x, stream=1), lambda: ops.embedding(ids, table, x, scale="two", stream=1),
           lambda: ops.embedding_backward(x, half, table, workspace=x, stream=1), lambda: ops.embedding_backward(here(6, 9), ids, table, workspace=x, stream=1),
           lambda: ops.embedding_backward(x, None, table, workspace=x, stream=1), lambda: ops.embedding_backward(x, ids, table, workspace=here(4), stream=1),
           lambda: ops.layernorm(x, v, None, y, stream=1), lambda: ops.layernorm(x, w, v, y, stream=1), lambda: ops.layernorm(x, w, w, y, mean=w, stream=1),
           lambda: ops.layernorm(x, w, w, y, residual=x, h=here(6, 8, dtype=torch.bfloat16), stream=1), lambda: ops.layernorm(x, w, w, here(8, 6).t(), stream=1),
           lambda: ops.layernorm_backward(x, y, w, v, w, x, stream=1), lambda: ops.layernorm_backward(x, y, w, v, v, here(6, 8, dtype=torch.bfloat16), stream=1),
           lambda: ops.layernorm_backward(x, y, w, v, v, x, w, workspace=here(4), stream=1),
           lambda: ops.token_logprobs(x, None, v, stream=1), lambda: ops.token_logprobs(x, half, v, stream=1), lambda: ops.token_logprobs(x, ids, w, stream=1),
           lambda: ops.token_logprobs(x, ids, v, top_values=tv, top_index=here(6, 2, dtype=torch.int32), stream=1), lambda: ops.token_logprobs(x, ids, v, top_index=tv, stream=1),
           lambda: ops.token_logprobs(x, ids, v, top_index=here(6, 0, dtype=torch.int32), stream=1), lambda: ops.token_logprobs(code, ids, v, stream=1),
           lambda: ops.token_logprobs_backward(x, None, v, y, dlogp=v, stream=1), lambda: ops.token_logprobs_backward(x, ids, None, y, dlogp=v, stream=1),
           lambda: ops.token_logprobs_backward(x, ids, v, y, dlogp=v, dentropy=v, stream=1), lambda: ops.token_logprobs_backward(x, ids, v, here(6, 9), dlogp=v, stream=1),
           lambda: ops.distill(x, at, tv, v, stream=1), lambda: ops.distill(x, wrong, wrong, v, stream=1), lambda: ops.distill(x, at, wrong, None, stream=1),
           lambda: ops.distill(x, at, wrong, w, stream=1), lambda: ops.distill_backward(x, at, wrong, None, v, y, stream=1),
           lambda: ops.distill_backward(x, at, wrong, v, None, y, stream=1), lambda: ops.distill_backward(x, at, wrong, v, v, code, stream=1),
           lambda: ops.token_logprobs(here(6, 16)[:, ::2], ids, v, stream=1), lambda: ops.distill(x, iv, here(6, 6)[:, ::2], v, stream=1)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"call {i} was not refused")


def test_binding_refuses_operands_of_different_devices(ops):
    here, there = (lambda *s, **k: _at("cuda:0", *s, **k)), (lambda *s, **k: _at("cuda:1", *s, **k))
    x, w, v, ids, at, tv, ti = here(8, 8), here(8), here(8), here(8, dtype=torch.int64), here(8, 3, dtype=torch.int32), here(8, 3), here(8, 3, dtype=torch.int32)
    far, fv, fids, fat, ftv = there(8, 8), there(8), there(8, dtype=torch.int64), there(8, 3, dtype=torch.int32), there(8, 3)
    for call in (lambda: ops.embedding(fids, x, x, stream=1), lambda: ops.embedding(ids, x, far, stream=1), lambda: ops.embedding_backward(far, ids, x, workspace=x, stream=1),
                 lambda: ops.embedding_backward(x, fids, x, workspace=x, stream=1), lambda: ops.layernorm(x, fv, w, x, stream=1), lambda: ops.layernorm(x, w, fv, x, stream=1),
                 lambda: ops.layernorm(x, w, w, far, stream=1), lambda: ops.layernorm(x, w, w, x, residual=far, stream=1), lambda: ops.layernorm(x, w, w, x, residual=x, h=far, stream=1),
                 lambda: ops.layernorm(x, w, w, x, mean=fv, stream=1), lambda: ops.layernorm(x, w, w, x, rstd=fv, stream=1), lambda: ops.layernorm_backward(far, x, w, v, v, x, stream=1),
                 lambda: ops.layernorm_backward(x, x, w, fv, v, x, stream=1), lambda: ops.layernorm_backward(x, x, w, v, fv, x, stream=1),
                 lambda: ops.layernorm_backward(x, x, w, v, v, far, stream=1), lambda: ops.layernorm_backward(x, x, w, v, v, x, dres=far, stream=1),
                 lambda: ops.layernorm_backward(x, x, w, v, v, x, fv, workspace=x, stream=1), lambda: ops.layernorm_backward(x, x, w, v, v, x, None, fv, workspace=x, stream=1),
                 lambda: ops.token_logprobs(x, fids, v, stream=1), lambda: ops.token_logprobs(x, ids, fv, stream=1), lambda: ops.token_logprobs(x, ids, v, lse=fv, stream=1),
                 lambda: ops.token_logprobs(x, ids, v, entropy=fv, stream=1), lambda: ops.token_logprobs(x, ids, v, top_values=ftv, top_index=ti, stream=1),
                 lambda: ops.token_logprobs(x, ids, v, top_values=tv, top_index=fat, stream=1), lambda: ops.token_logprobs_backward(x, fids, v, x, dlogp=v, stream=1),
                 lambda: ops.token_logprobs_backward(x, ids, fv, x, dlogp=v, stream=1), lambda: ops.token_logprobs_backward(x, ids, v, far, dlogp=v, stream=1),
                 lambda: ops.token_logprobs_backward(x, ids, v, x, dlogp=fv, stream=1), lambda: ops.token_logprobs_backward(x, ids, v, x, dlse=fv, stream=1),
                 lambda: ops.token_logprobs_backward(x, ids, v, x, dentropy=fv, entropy=v, stream=1), lambda: ops.token_logprobs_backward(x, ids, v, x, dentropy=v, entropy=fv, stream=1),
                 lambda: ops.distill(x, fat, tv, v, stream=1), lambda: ops.distill(x, at, ftv, v, stream=1), lambda: ops.distill(x, at, tv, fv, stream=1),
                 lambda: ops.distill(x, at, tv, v, lse=fv, stream=1), lambda: ops.distill_backward(x, at, tv, fv, v, x, stream=1),
                 lambda: ops.distill_backward(x, at, tv, v, fv, x, stream=1), lambda: ops.distill_backward(x, at, tv, v, v, far, stream=1)):
        with pytest.raises(ValueError, match="different devices"):
            call()
    for call in (lambda: ops.embedding_backward(x, ids, x, workspace=there(1 << 16), stream=1), lambda: ops.layernorm_backward(x, x, w, v, v, x, v, workspace=there(1 << 16), stream=1)):
        with pytest.raises(ValueError, match="operands' GPU"):
            call()
