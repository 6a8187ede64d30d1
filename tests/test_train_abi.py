"""The operators of a training step without a GPU: bad arguments are refused synchronously with
the documented status, before any HIP call, and size queries answer."""
import ctypes
import random

import pytest

from paper_2411_10764_amd import ml2

OK, INVALID, UNSUPPORTED = ml2.ML2_OK, ml2.ML2_ERR_INVALID_ARG, ml2.ML2_ERR_UNSUPPORTED
F32, BF16, F16 = ml2.ML2_F32, ml2.ML2_BF16, ml2.ML2_F16
MB = 1 << 20  # addresses, far apart, that nothing here reads
X, D, W, B, M, R, O, GW, GB, WS = (i * 16 * MB for i in range(1, 11))
BIG = 1 << 24
INF, NAN = float("inf"), float("nan")


def _norm(dtype=F32, x=X, rows=3, width=8, ld=8, pd=F32, w=W, b=B, eps=1e-5, out=O, out_ld=8,
          mean=M, rstd=R):
    return ml2.lib().ml2_layer_norm(dtype, x, rows, width, ld, pd, w, b, eps, out, out_ld, mean,
                                    rstd, None)


def _grad(dtype=F32, x=X, rows=3, width=8, ld=8, dout=D, dout_ld=8, pd=F32, w=W, mean=M, rstd=R,
          dx=O, dx_ld=8, gd=F32, dw=GW, db=GB, ws=WS, ws_bytes=BIG):
    return ml2.lib().ml2_layer_norm_grad(dtype, x, rows, width, ld, dout, dout_ld, pd, w, mean,
                                         rstd, dx, dx_ld, gd, dw, db, ws, ws_bytes, None)


ROWS = [dict(dtype=3), dict(dtype=-1), dict(pd=7), dict(dtype=BF16, pd=F16), dict(dtype=F32, pd=BF16),
        dict(x=None), dict(rows=-1), dict(rows=1 << 31), dict(width=-1), dict(ld=7),
        dict(ld=(1 << 32) + 1), dict(x=X + 2), dict(dtype=F16, x=X + 1), dict(w=W + 2)]


@pytest.mark.parametrize("bad", ROWS + [
    dict(out=None), dict(out_ld=7), dict(out_ld=(1 << 32) + 1), dict(out=O + 2), dict(b=B + 1),
    dict(mean=M + 2), dict(rstd=R + 1), dict(eps=0.0), dict(eps=-1e-5), dict(eps=NAN),
    dict(eps=INF),
    # memory that is shared: the output over its rows, one another and the parameters
    dict(out=X + 4), dict(out=X + 4 * 8), dict(out=X, out_ld=9), dict(mean=R), dict(rstd=M + 8),
    dict(mean=O), dict(mean=X + 40), dict(rstd=O + 92), dict(w=O), dict(b=O + 64), dict(w=M),
    dict(b=R + 8), dict(x=X, ld=16, out=X + 4 * 7, out_ld=16)])
def test_layer_norm_refuses(bad):
    assert _norm(**bad) == INVALID and ml2.lib().ml2_last_error()


@pytest.mark.parametrize("bad", [b for b in ROWS] + [
    dict(dout=None), dict(mean=None), dict(rstd=None), dict(dout_ld=7), dict(dx_ld=7),
    dict(dout_ld=(1 << 32) + 1), dict(dx_ld=(1 << 32) + 1), dict(gd=9), dict(gd=BF16),
    dict(dtype=BF16, gd=F16), dict(dout=D + 1), dict(dx=O + 2), dict(mean=M + 2), dict(rstd=R + 2),
    dict(dw=GW + 2), dict(db=GB + 1), dict(ws=None), dict(ws=WS + 128), dict(ws_bytes=0),
    dict(ws_bytes=8 * 4),
    dict(dx=X + 4), dict(dx=X, dx_ld=9), dict(dx=D + 8 * 4), dict(dx=W), dict(dx=M), dict(dx=WS),
    dict(dw=GB), dict(dw=GB + 28), dict(dw=X), dict(db=D + 92), dict(dw=W), dict(db=M), dict(db=R),
    dict(dw=O), dict(dw=WS), dict(ws=X), dict(ws=D), dict(ws=M), dict(ws=R), dict(ws=W)])
def test_layer_norm_grad_refuses(bad):
    assert _grad(**bad) == INVALID and ml2.lib().ml2_last_error()


def test_widths_beyond_the_limit():
    assert _norm(width=65537, ld=65537, out_ld=65537) == UNSUPPORTED
    assert _grad(width=65537, ld=65537, dout_ld=65537, dx_ld=65537) == UNSUPPORTED
    size = ctypes.c_size_t()
    f = ml2.lib().ml2_layer_norm_grad_workspace_bytes
    assert f(3, 65537, ctypes.byref(size)) == UNSUPPORTED
    for rows, width in ((-1, 3), (3, -1), (1 << 31, 3), (3, 1 << 31)):
        assert f(rows, width, ctypes.byref(size)) == INVALID
    assert f(3, 3, None) == INVALID


def test_nothing_to_do_asks_for_nothing():
    assert _norm(rows=0, x=None, out=None, mean=None, rstd=None) == OK
    assert _norm(width=0, ld=0, out_ld=0, x=None, out=None, w=None, b=None) == OK
    assert _grad(width=0, ld=0, dout_ld=0, dx_ld=0, x=None, dout=None, dx=None) == OK
    assert _grad(dx=None, dw=None, db=None) == OK
    assert _grad(rows=0, dw=None, db=None, x=None, dout=None, mean=None, rstd=None) == OK


def test_workspaces_grow_with_the_sizes_they_are_for():
    for width in (1, 100, 1000, 5000, 16384, 16385, 65536):
        sizes = [ml2.ml2_layer_norm_grad_workspace_bytes(r, width) for r in (0, 1, 10, 1000, 10 ** 6)]
        assert sizes[0] == 0 and sizes[1] >= 8 * width and sizes == sorted(sizes)
    # the parts of the parameters' sums stay small beside the rows
    assert ml2.ml2_layer_norm_grad_workspace_bytes(10 ** 6, 1024) <= 16 << 20


# ---- norms -------------------------------------------------------------------------

def _norms(dtype=F32, grads=(X, D), sizes=(100, 50), count=None, scale=1.0, limit=1.0, norm=M,
           factor=R, step=B, ws=WS, ws_bytes=BIG):
    g = None if grads is None else (ctypes.c_void_p * len(grads))(*grads)
    s = None if sizes is None else (ctypes.c_int64 * len(sizes))(*sizes)
    return ml2.lib().ml2_grad_norm(dtype, g, s, len(sizes or ()) if count is None else count, scale,
                                   limit, norm, factor, step, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(grads=None), dict(sizes=None, count=2), dict(count=-1),
    dict(sizes=(100, -1)), dict(grads=(X, None)), dict(grads=(X, D + 2)), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(limit=0.0), dict(limit=-1.0),
    dict(limit=NAN), dict(norm=M + 2), dict(factor=R + 1), dict(step=B + 2), dict(ws=None),
    dict(ws=WS + 8), dict(ws_bytes=8), dict(norm=R), dict(step=M), dict(norm=X + 396),
    dict(factor=D), dict(step=D + 196), dict(ws=X), dict(ws=D), dict(norm=WS + 8)])
def test_grad_norm_refuses(bad):
    assert _norms(**bad) == INVALID and ml2.lib().ml2_last_error()


def test_grad_norm_limits():
    assert _norms(sizes=(100, (1 << 40) + 1)) == UNSUPPORTED
    assert _norms(count=65537) == UNSUPPORTED
    assert _norms(norm=None, factor=None, step=None) == OK
    size = ctypes.c_size_t()
    f = ml2.lib().ml2_grad_norm_workspace_bytes
    sizes = (ctypes.c_int64 * 2)(5, -1)
    assert f(sizes, 2, ctypes.byref(size)) == INVALID
    assert f(None, 2, ctypes.byref(size)) == INVALID
    assert f(sizes, 1, None) == INVALID
    assert f(sizes, -1, ctypes.byref(size)) == INVALID
    assert f(sizes, 65537, ctypes.byref(size)) == UNSUPPORTED
    assert ml2.ml2_grad_norm_workspace_bytes([1 << 40] * 100) < 1 << 20


# ---- AdamW ------------------------------------------------------------------------------

N = 1000
FIELDS = dict(param=X, grad=D, m=M, v=R, param_out=None, m_out=None, v_out=None, copy=None, n=N,
              weight_decay=0.1)


def _adamw(pd=F32, gd=F32, bits=32, tensors=None, count=None, options=None, no_options=False,
           second=None, **first):
    o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    o.update(options or {})
    rows = [dict(FIELDS, **first)] + ([] if second is None else [dict(FIELDS, **second)])
    a = (ml2.ml2_adamw_tensor * len(rows))(*[ml2.ml2_adamw_tensor(**r) for r in rows])
    op = ml2.ml2_adamw_options(**o)
    return ml2.lib().ml2_adamw(pd, gd, bits, None if tensors == 0 else a,
                               len(rows) if count is None else count,
                               None if no_options else ctypes.byref(op), None)


@pytest.mark.parametrize("bad", [
    dict(pd=3), dict(gd=-1), dict(bits=16), dict(bits=0), dict(tensors=0), dict(count=-1),
    dict(no_options=True), dict(param=None), dict(grad=None), dict(m=None), dict(v=None),
    dict(n=-1), dict(weight_decay=NAN), dict(weight_decay=INF), dict(param=X + 2),
    dict(gd=BF16, grad=D + 1), dict(m=M + 2), dict(v=R + 1), dict(bits=8, m=M + 2),
    dict(param_out=O + 2), dict(m_out=O + 2), dict(v_out=O + 1), dict(gd=F16, copy=O + 1)] + [
    dict(options=o) for o in (
        dict(lr=NAN), dict(lr=INF), dict(lr=1e39), dict(beta1=-0.1), dict(beta1=1.0),
        dict(beta1=NAN), dict(beta2=1.0), dict(beta2=-1e-9), dict(eps=0.0), dict(eps=-1.0),
        dict(eps=NAN), dict(eps=1e-60), dict(eps=1e-39), dict(eps=1e60), dict(step=0), dict(step=-1),
        dict(step=1 << 31), dict(lr_device=B + 2), dict(step_device=B + 1), dict(factor=B + 2),
        # an option in memory that the step writes
        dict(lr_device=X), dict(step_device=M + 4 * N - 4), dict(factor=R + 40))] + [
    # arrays that are written and shared
    dict(m=X), dict(v=M), dict(v=M + 4 * N - 4), dict(grad=X), dict(grad=M + 4), dict(copy=D),
    dict(copy=X), dict(copy=M), dict(param_out=X + 4), dict(param_out=D), dict(param_out=M),
    dict(m_out=R), dict(m_out=O, v_out=O + 4 * N - 4), dict(v_out=R + 8),
    dict(m_out=X), dict(bits=8, v=M + 1036), dict(bits=8, v=M + 4 * 260 - 4),
    dict(second={}), dict(second=dict(m=O, v=GW, grad=GB)),
    dict(second=dict(param=O, m=GW, v=GB, grad=X)), dict(second=dict(param=O, m=GW, v=M + 400)),
    # the first tensor's old parameters, which stay as they were, are the second's new ones
    dict(param_out=B, second=dict(param=O, m=GW, v=GB, param_out=X))])
def test_adamw_refuses(bad):
    assert _adamw(**bad) == INVALID and ml2.lib().ml2_last_error()


def test_adamw_limits():
    assert _adamw(n=(1 << 40) + 1) == UNSUPPORTED
    assert _adamw(count=65537) == UNSUPPORTED
    assert _adamw(n=0, param=None, grad=None, m=None, v=None) == OK
    assert _adamw(tensors=0, count=0) == OK


def test_state_sizes():
    for n, want in ((0, 0), (1, 260), (256, 260), (257, 520), (1 << 33, (1 << 33) + (1 << 27))):
        assert ml2.ml2_adamw_state_bytes(8, n) == want
        assert ml2.ml2_adamw_state_bytes(32, n) == 4 * n
    size = ctypes.c_size_t()
    f = ml2.lib().ml2_adamw_state_bytes
    assert f(16, 5, ctypes.byref(size)) == INVALID and f(8, -1, ctypes.byref(size)) == INVALID
    assert f(8, 5, None) == INVALID and f(8, (1 << 40) + 1, ctypes.byref(size)) == UNSUPPORTED


def test_the_binding_refuses():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device"):
        ml2.ml2_layer_norm(x, None, None, torch.zeros(4, 8))
    with pytest.raises(ValueError, match="device"):
        ml2.ml2_layer_norm_grad(x, x, None, x, x, x)
    for make in (lambda: ml2.GradNorm([x]), lambda: ml2.AdamW([x], [x])):
        with pytest.raises(ValueError, match="device"):
            make()
    for make in (lambda: ml2.GradNorm([]), lambda: ml2.AdamW([], [])):
        with pytest.raises(ValueError, match="hold"):
            make()


# ---- memory between the rows ---------------------------------------------------------

@pytest.mark.parametrize("name", ["x", "dout"])
def test_a_workspace_meets_rows_only_in_their_elements(name):
    """A call that has nothing to write ends after its checks: OK where the workspace has no
    element of the rows, between them too, and refused where it has one."""
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        dtype, size = rng.choice(((F32, 4), (BF16, 2), (F16, 2)))
        rows, width = rng.randint(0, 6), rng.randint(1, 7)
        need = ml2.ml2_layer_norm_grad_workspace_bytes(rows, width)
        ld = width + rng.randint(0, 3 * need // size + 4)
        off = rng.randint(-(rows * ld + 10), need // size + 10)
        at = WS + off * size
        used = {at + r * ld * size + i for r in range(rows) for i in range(width * size)}
        want = any(WS <= b < WS + need for b in used)
        rest = dict(dict(ld=8, dout_ld=8), **{name: at, "ld" if name == "x" else "dout_ld": ld})
        got = _grad(dtype, rows=rows, width=width, pd=dtype, gd=dtype, dx=None, dw=None, db=None,
                    ws_bytes=need, **rest)
        assert got == (INVALID if want else OK), (dtype, rows, width, ld, off)
        seen[want] += 1
    assert min(seen.values()) > 500


FAR = dict(rows=(1 << 31) - 1, width=8, ld=1 << 32)  # the last row lies beyond 64 bits
PITCH, P = 1 << 34, 1 << 40


@pytest.mark.parametrize("at", [P, P + 28, P - 4 * FAR["rows"] + 4, P + PITCH, P + 2 * PITCH + 28])
def test_statistics_in_rows_that_reach_far(at):
    """No other two arrays meet: out's rows lie behind the statistics' 8.6 GB."""
    for name in ("mean", "rstd"):
        assert _norm(**FAR, **dict(dict(x=P, w=None, b=None, mean=None, rstd=None), out=P + (3 << 32),
                                   out_ld=1 << 32, **{name: at})) == INVALID
        assert "shares memory" in ml2.lib().ml2_last_error().decode()


@pytest.mark.parametrize("bad", [
    dict(dw=P + 7 * PITCH), dict(dw=P + 7 * PITCH + 64 + 28), dict(db=P + 7 * PITCH + 28),
    dict(ws=P + 5 * PITCH), dict(dx=P + 3 * PITCH + 512, dx_ld=1 << 32, dw=P + 9 * PITCH + 512)])
def test_sums_and_a_workspace_in_rows_that_reach_far(bad):
    args = dict(x=P, dout=P + 64, dout_ld=1 << 32, w=None, mean=P + 1024, rstd=P + PITCH + 1024,
                dx=None, dw=None, db=None, ws=P + 5 * PITCH + 256)
    assert _grad(**FAR, **dict(args, **bad)) == INVALID
    assert "shares memory" in ml2.lib().ml2_last_error().decode()
