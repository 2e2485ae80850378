"""Host side of the operators around the GEMMs, no GPU: struct layouts, workspace sizes, and the refusals, which come
before anything touches a device (the addresses below are never dereferenced)."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVAL, UNSUPPORTED, CUDA = -1, -2, -6


@pytest.fixture(scope="module")
def ops():
    import paper_2512_22142_b200 as cl
    return cl.ops


def test_struct_layouts_match_the_header(ops, tmp_path):
    names = {"adamw_tensor": ops._AdamwTensor, "adamw_step": ops._AdamwStep, "rmsnorm": ops._Rmsnorm, "rmsnorm_backward": ops._RmsnormBackward,
             "linear": ops._Linear, "act_backward": ops._ActBackward}
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


def _refused(rc, code=INVAL):
    assert rc == code


def _norm(ops, **kw):
    d = ops._Rmsnorm()
    base = dict(rows=4, cols=8, eps=1e-5, x_type=1, x=4096, ldx=8, y_type=1, y=8192, ldy=8)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return ops.lib.cleave_rmsnorm(ctypes.byref(d), None)


@pytest.mark.parametrize("kw", [dict(cols=0), dict(x=None), dict(x_type=0), dict(x_type=3), dict(ldx=7), dict(x=4097), dict(y_type=3),
                                dict(scale=4096), dict(y_type=3, scale=4097), dict(h=4096, ldh=8), dict(r=4096), dict(r_type=1, r=4096, ldr=4),
                                dict(r_type=2, r=4098, ldr=8), dict(w=4096), dict(w_type=3, w=4096), dict(rstd=4098), dict(eps=-1.0),
                                dict(eps=float("nan")), dict(y=None), dict(ldy=1 << 41), dict(r_type=1, r=4096, ldr=8, h=4097, ldh=8)])
def test_rmsnorm_refuses(ops, kw):
    _refused(_norm(ops, **kw))


def test_rmsnorm_limits(ops):
    assert _norm(ops, rows=0, x=None, y=None) == 0
    _refused(_norm(ops, rows=1 << 31), UNSUPPORTED)
    assert ops.lib.cleave_rmsnorm(None, None) == INVAL


def _norm_bwd(ops, ws=4096, **kw):
    d = ops._RmsnormBackward()
    base = dict(rows=4, cols=8, dy_type=1, dy=4096, lddy=8, h_type=1, h=8192, ldh=8, rstd=4096, dx=16384, lddx=8, dw=4096)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return ops.lib.cleave_rmsnorm_backward(ctypes.byref(d), ws, None)


@pytest.mark.parametrize("kw", [dict(cols=0), dict(dy=None), dict(dy_type=3), dict(lddy=4), dict(h_type=0), dict(h=8193), dict(dx=None), dict(lddx=7),
                                dict(rstd=None), dict(rstd=4098), dict(ws=None), dict(ws=4100), dict(dres=4097, lddres=8), dict(dres=4096, lddres=2),
                                dict(dw=4098), dict(w=4096)])
def test_rmsnorm_backward_refuses(ops, kw):
    _refused(_norm_bwd(ops, **kw))


def _linear(ops, **kw):
    d = ops._Linear()
    base = dict(in_type=1, c_type=1, A=4096, B=8192, C=16384, ldc=32)
    g = dict(M=8, N=32, K=64, lda=64, ldb=32, transA=0, transB=0)
    for k, v in {**base, **kw}.items():
        if k in g:
            g[k] = v
        else:
            setattr(d, k, v)
    for k, v in g.items():
        setattr(d.g, k, v)
    return ops.lib.cleave_linear(ctypes.byref(d), None)


@pytest.mark.parametrize("kw", [dict(N=0), dict(K=0), dict(in_type=2), dict(in_type=0), dict(c_type=3), dict(c_type=0), dict(act=5), dict(A=None),
                                dict(A=4104), dict(B=8200), dict(lda=60), dict(lda=56), dict(ldb=24), dict(transB=1), dict(transA=2), dict(C=None), dict(ldc=31),
                                dict(C=16385), dict(bias=4096), dict(bias_type=1, bias=4097), dict(z_type=2, z=4096, ldz=16), dict(mul_type=3, mul=4096, ldmul=32),
                                dict(res_type=1, ldres=32), dict(scale_a=4098), dict(scale_b=4097), dict(M=1 << 31)])
def test_linear_refuses(ops, kw):
    _refused(_linear(ops, **kw))


def test_linear_limits(ops):
    assert _linear(ops, M=0, A=None, C=None) == 0
    _refused(_linear(ops, in_type=3), UNSUPPORTED)                                   # E4M3 needs both operands K-contiguous
    _refused(_linear(ops, in_type=3, transB=1, ldb=72))                              # 16-byte rows


def _act(ops, ws=4096, **kw):
    d = ops._ActBackward()
    base = dict(rows=4, cols=8, act=2, dy_type=1, dy=4096, lddy=8, z_type=1, z=8192, ldz=8, dz_type=1, dz=16384, lddz=8, dbias=4096)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return ops.lib.cleave_act_backward(ctypes.byref(d), ws, None)


@pytest.mark.parametrize("kw", [dict(cols=0), dict(act=9), dict(dy=None), dict(dy_type=3), dict(lddy=7), dict(z=None), dict(z_type=0, z=None), dict(ldz=1),
                                dict(dz_type=0), dict(dz=16385), dict(mul_type=1), dict(dmul_type=1, dmul=4096), dict(ws=None), dict(ws=4104), dict(dbias=4097),
                                dict(act=0, z_type=0, z=None, dmul_type=1, dmul=4096, lddmul=8)])
def test_act_backward_refuses(ops, kw):
    _refused(_act(ops, **kw))


def _create(ops, n=1, state=2, grad=2, **kw):
    t = (ops._AdamwTensor * 1)()
    base = dict(numel=512, p=4096, g=8192, m=16384, v=32768)
    for k, v in {**base, **kw}.items():
        setattr(t[0], k, v)
    h = ctypes.c_void_p()
    rc = ops.lib.cleave_adamw_create(t, n, state, grad, ctypes.byref(h))
    assert rc != 0 and not h.value
    return rc


@pytest.mark.parametrize("kw", [dict(n=0), dict(state=1), dict(state=0), dict(grad=3), dict(grad=0), dict(p=None), dict(p=4098), dict(g=None), dict(g=8193),
                                dict(m=None), dict(v=32770), dict(w=4097), dict(numel=1 << 41), dict(weight_decay=float("nan")),
                                dict(state=3), dict(state=3, m_scale=4096), dict(state=3, m_scale=4096, v_scale=4098), dict(m_scale=4096, v_scale=4096)])
def test_adamw_refuses(ops, kw):
    _refused(_create(ops, **kw))


def test_adamw_step_refuses_a_missing_handle(ops):
    s = ops._AdamwStep()
    assert ops.lib.cleave_adamw_step(None, ctypes.byref(s), None) == INVAL
    assert ops.lib.cleave_adamw_set_grads(None, None, None) == INVAL
    ops.lib.cleave_adamw_destroy(None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="what a machine without a GPU answers")
def test_without_a_device_the_calls_say_so(ops):
    assert _norm(ops) == CUDA and _norm_bwd(ops) == CUDA and _linear(ops) == CUDA and _act(ops) == CUDA and _create(ops) == CUDA


def test_workspaces(ops):
    for fn in (ops.rmsnorm_backward_workspace, ops.act_backward_workspace):
        assert fn(0, 100) == 0 and fn(1, 100) >= 400
        assert fn(1 << 31, 100) <= 100 * 4 * 4096              # bounded: partial sums, not rows


def test_binding_refuses_what_the_library_cannot_see(ops):
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    w = torch.zeros(8)
    for call in (lambda: ops.rmsnorm(x, w, x), lambda: ops.rmsnorm(x[0], w, x), lambda: ops.linear(x, x, x, transB=True),
                 lambda: ops.act_backward(x, x, x, act="relu"), lambda: ops.quantize_rows(x, x, w), lambda: ops.rmsnorm_backward(x, x, w, w, x),
                 lambda: ops.AdamW([], [], [], []), lambda: ops.AdamW([w], [w], [w], [w]), lambda: ops.AdamW([w], [x], [x], [w])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("raw", [False, True])
def test_a_workspace_for_another_stream_comes_from_that_streams_pool(ops, monkeypatch, raw):
    """The allocator hands out blocks in the order of the stream that is current when it is asked: a block for a launch on
    another stream is asked for with that stream current, or work still pending on the first one may use it too."""
    import contextlib

    class Stream:
        cuda_stream = 77

    current, asked = [], []

    @contextlib.contextmanager
    def stream_context(s):
        current.append(s)
        yield
        current.pop()

    real = torch.empty

    def empty(*size, **kw):
        asked.append(current[-1].cuda_stream if current else None)
        t = real(*size, **kw)
        t.record_stream = lambda s: None
        return t

    def external(handle, device=None):
        s = Stream()
        s.cuda_stream = handle
        return s
    monkeypatch.setattr(torch.cuda, "stream", stream_context)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch, "empty", empty)
    ws = ops._workspace(None, 400, torch.zeros(1), 78 if raw else Stream())
    assert ws.numel() == 400 and asked == [78 if raw else 77] and not current
    assert ops._workspace(ws, 400, ws, Stream()) is ws and ops._workspace(None, 400, ws, None) is None and len(asked) == 1


def test_binding_refuses_operands_of_different_devices(ops):
    """Tensors without memory that say they are on one GPU or another: the refusal comes before anything else."""
    from torch._subclasses.fake_tensor import FakeTensorMode

    def at(device, *size, dtype=torch.float32):
        with FakeTensorMode():
            return torch.empty(*size, dtype=dtype, device=device)
    here, there = (lambda *s, **k: at("cuda:0", *s, **k)), (lambda *s, **k: at("cuda:1", *s, **k))
    x, w, v = here(8, 8), here(8), here(8)
    code, bf = here(8, 8, dtype=torch.float8_e4m3fn), here(8, 8, dtype=torch.bfloat16)
    far, fv, fbf = there(8, 8), there(8), there(8, 8, dtype=torch.bfloat16)
    ws, fws = here(1 << 16, dtype=torch.uint8), there(1 << 16, dtype=torch.uint8)
    for call in (lambda: ops.rmsnorm(x, fv, x, stream=1), lambda: ops.rmsnorm(x, w, far, stream=1), lambda: ops.rmsnorm(x, w, x, residual=far, stream=1),
                 lambda: ops.rmsnorm(x, w, x, residual=x, h=far, stream=1), lambda: ops.rmsnorm(x, w, x, rstd=fv, stream=1),
                 lambda: ops.rmsnorm(x, w, code, scale=fv, stream=1), lambda: ops.quantize_rows(far, code, v, stream=1),
                 lambda: ops.quantize_rows(x, code, fv, stream=1), lambda: ops.rmsnorm_backward(far, x, w, v, x, stream=1),
                 lambda: ops.rmsnorm_backward(x, x, w, fv, x, stream=1), lambda: ops.rmsnorm_backward(x, x, w, v, far, stream=1),
                 lambda: ops.rmsnorm_backward(x, x, w, v, x, fv, workspace=ws, stream=1), lambda: ops.rmsnorm_backward(x, x, w, v, x, dres=far, stream=1),
                 lambda: ops.linear(bf, fbf, x, stream=1), lambda: ops.linear(bf, bf, far, stream=1), lambda: ops.linear(bf, bf, x, bias=fv, stream=1),
                 lambda: ops.linear(bf, bf, x, scale_a=fv, stream=1), lambda: ops.linear(bf, bf, x, scale_b=fv, stream=1),
                 lambda: ops.linear(bf, bf, x, z=far, stream=1), lambda: ops.linear(bf, bf, x, mul=far, stream=1),
                 lambda: ops.linear(bf, bf, x, residual=far, stream=1), lambda: ops.act_backward(x, far, x, act="relu", stream=1),
                 lambda: ops.act_backward(x, x, far, act="relu", stream=1), lambda: ops.act_backward(x, x, x, act="relu", mul=far, stream=1),
                 lambda: ops.act_backward(x, x, x, act="relu", dmul=far, stream=1),
                 lambda: ops.act_backward(x, x, x, act="relu", dbias=fv, workspace=ws, stream=1)):
        with pytest.raises(ValueError, match="different devices"):
            call()
    for call in (lambda: ops.act_backward(x, x, x, act="relu", dbias=v, workspace=fws, stream=1),
                 lambda: ops.rmsnorm_backward(x, x, w, v, x, v, workspace=fws, stream=1)):
        with pytest.raises(ValueError, match="operands' GPU"):
            call()


def _bare_optimizer(ops, monkeypatch, device, calls, during=lambda: None):
    """An AdamW of `device` without memory or library behind it; every library call is noted with its current device."""
    import contextlib
    from types import SimpleNamespace
    current = [0]

    @contextlib.contextmanager
    def on(d):
        current.append(d)
        yield
        current.pop()

    def step(h, s, stream):
        during()
        r = s._obj
        calls.append(("step", current[-1], stream, r.lr, r.step, r.seed))
        return 0

    def set_grads(h, ptrs, stream):
        calls.append(("set_grads", current[-1], stream))
        return 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[-1])
    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(ops, "lib", SimpleNamespace(cleave_adamw_step=step, cleave_adamw_set_grads=set_grads, cleave_adamw_destroy=lambda h: None))
    opt = object.__new__(ops.AdamW)
    opt.__dict__.update(_h=0, _n=0, _grad=2, _device=device, _keep=([], [], [], [], []))
    return opt


def test_adamw_steps_on_its_own_device(ops, monkeypatch):
    """Like every other operator: whatever device is the current one."""
    for device in (0, 1):
        calls = []
        opt = _bare_optimizer(ops, monkeypatch, device, calls)
        opt.step(step=3, lr=0.5, seed=9, stream=5)
        opt.set_grads([], stream=5)
        assert calls == [("step", device, 5, 0.5, 3, 9), ("set_grads", device, 5)]


def test_adamw_steps_from_two_threads_keep_their_arguments(ops, monkeypatch):
    """A library call releases the interpreter: another thread's step of the same optimizer may begin while it runs."""
    import threading
    calls, inner = [], []

    def during():
        if not inner:                          # inside the first call, another thread steps
            t = threading.Thread(target=lambda: opt.step(step=8, lr=0.25, seed=2, stream=6))
            inner.append(t)
            t.start()
            t.join()
    opt = _bare_optimizer(ops, monkeypatch, 0, calls, during)
    opt.step(step=7, lr=0.5, seed=1, stream=5)
    assert sorted(calls) == [("step", 0, 5, 0.5, 7, 1), ("step", 0, 6, 0.25, 8, 2)]


@pytest.mark.parametrize("cols", [1 << 31, (1 << 32) - 200, (1 << 32) - 1])
def test_columns_beyond_31_bits_are_refused(ops, cols):
    """The kernels count columns in 32 bits, in steps of a CTA's threads."""
    ld = 1 << 33
    _refused(_norm(ops, cols=cols, ldx=ld, ldy=ld), UNSUPPORTED)
    _refused(_norm_bwd(ops, cols=cols, lddy=ld, ldh=ld, lddx=ld), UNSUPPORTED)
    _refused(_act(ops, cols=cols, lddy=ld, ldz=ld, lddz=ld), UNSUPPORTED)
    _refused(ops.lib.cleave_quantize_rows(4096, 1, 4, cols, ld, 8192, ld, 4096, None), UNSUPPORTED)


def test_marshalling_is_rebuilt_for_another_torch(monkeypatch, tmp_path):
    """The extension is bound to torch's binary interface: one built against another version is stale, whatever its date."""
    from paper_2512_22142_b200 import build
    path = tmp_path / "_marshal.so"
    monkeypatch.setattr(build, "MARSHAL_PATH", str(path))
    assert build._marshal_is_stale()
    path.write_text("")
    os.utime(path, (2 ** 31, 2 ** 31))
    stamp = tmp_path / "_marshal.so.torch"
    assert build._marshal_is_stale()
    stamp.write_text(torch.__version__)
    assert not build._marshal_is_stale()
    stamp.write_text("2.0.0")
    assert build._marshal_is_stale()


def test_adamw_tensors_that_are_missing(ops, monkeypatch):
    """A tensor may go without a copy (None in its place); everything else is wanted for each tensor, and said so."""
    from types import SimpleNamespace

    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        f, code = (lambda n: torch.empty(n, device="cuda:0")), (lambda n: torch.empty(n, dtype=torch.float8_e4m3fn, device="cuda:0"))
        p, q, w = f(300), f(5), torch.empty(5, dtype=torch.bfloat16, device="cuda:0")
        made = []

        def create(table, n, state, grad, h):
            made.append([(r.numel, r.w) for r in table])
            return -1
        monkeypatch.setattr(ops, "lib", SimpleNamespace(cleave_adamw_create=create, cleave_strerror=lambda c: b"", cleave_adamw_destroy=lambda h: None))
        import contextlib
        monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
        import paper_2512_22142_b200 as cl
        with pytest.raises(cl.CleaveError):
            ops.AdamW([p, q], [p, q], [p, q], [p, q], copies=[None, w])
        assert [n for n, _ in made[0]] == [300, 5] and made[0][0][1] is None
        for bad in (lambda: ops.AdamW([p, None], [p, q], [p, q], [p, q]), lambda: ops.AdamW([p, q], [p, None], [p, q], [p, q]),
                    lambda: ops.AdamW([p, q], [p, q], [p, None], [p, q]), lambda: ops.AdamW([p, q], [p, q], [p, q], [None, q]),
                    lambda: ops.AdamW([None], [p], [p], [p]), lambda: ops.AdamW([p], [None], [p], [p]), lambda: ops.AdamW([p], [p], [None], [p]),
                    lambda: ops.AdamW([p], [p], [code(300)], [code(300)], m_scales=[None], v_scales=[f(2)])):
            with pytest.raises(ValueError):
                bad()
        assert len(made) == 1
