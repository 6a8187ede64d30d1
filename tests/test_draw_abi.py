"""The operators over rows of scores and over tables without a GPU: bad
arguments are refused synchronously with the documented status, before any
HIP call, and workspace queries answer."""
import ctypes

import pytest

from paper_2411_10764_amd import ml2

OK, INVALID, UNSUPPORTED = ml2.ML2_OK, ml2.ML2_ERR_INVALID_ARG, ml2.ML2_ERR_UNSUPPORTED
A = 0x10000  # an aligned address that nothing here reads
BIG = 1 << 40


def _sample(dtype=0, scores=A, n=10, ld=10, rows=2, valid=None, valid_ld=0, u=A, draws=3, idx=A,
            logprob=A, ws=A, ws_bytes=BIG):
    return ml2.lib().ml2_sample(dtype, scores, n, ld, rows, valid, valid_ld, None, None, None,
                                None, u, draws, idx, logprob, ws, ws_bytes, None)


def _logprob(dtype=0, scores=A, n=10, ld=10, rows=2, valid=None, valid_ld=0, targets=A, per_row=3,
             logprob=A, ws=A, ws_bytes=BIG):
    return ml2.lib().ml2_logprob(dtype, scores, n, ld, rows, valid, valid_ld, None, targets,
                                 per_row, logprob, ws, ws_bytes, None)


def _grad(dtype=0, scores=A, n=10, ld=10, rows=2, valid=None, valid_ld=0, targets=A, weight=A,
          per_row=3, logprob=A, grad=A, grad_ld=10, ws=A, ws_bytes=BIG):
    return ml2.lib().ml2_logprob_grad(dtype, scores, n, ld, rows, valid, valid_ld, None, targets,
                                      weight, per_row, logprob, grad, grad_ld, ws, ws_bytes, None)


def _embed(dtype=0, table=A, V=5, D=4, ld=4, ids=A, n=3, out=A, out_ld=4):
    return ml2.lib().ml2_embed(dtype, table, V, D, ld, ids, n, 1.0, out, out_ld, None)


def _embed_grad(dtype=1, dout=A, n=3, D=4, dout_ld=4, ids=A, grad_dtype=0, grad=A, V=5, grad_ld=4,
                ws=A, ws_bytes=BIG):
    return ml2.lib().ml2_embed_grad(dtype, dout, n, D, dout_ld, ids, 1.0, grad_dtype, grad, V,
                                    grad_ld, ws, ws_bytes, None)


ROWS = [dict(dtype=3), dict(dtype=-1), dict(scores=None), dict(n=-1), dict(n=1 << 31, ld=1 << 31),
        dict(ld=9), dict(rows=-1), dict(valid=A, valid_ld=9), dict(valid=A, valid_ld=-1),
        dict(ws=None), dict(ws=A + 128), dict(ws_bytes=0), dict(scores=A + 2), dict(scores=A + 1, dtype=1)]


@pytest.mark.parametrize("call,bad,status", [
    (_sample, b, INVALID) for b in ROWS + [dict(u=None), dict(idx=None), dict(logprob=None),
                                           dict(draws=-1)]] + [
    (_sample, dict(draws=16385), UNSUPPORTED), (_sample, dict(rows=2097153), UNSUPPORTED)] + [
    (_logprob, b, INVALID) for b in ROWS + [dict(targets=None), dict(logprob=None),
                                            dict(per_row=-1)]] + [
    (_logprob, dict(per_row=16385), UNSUPPORTED)] + [
    (_grad, b, INVALID) for b in ROWS + [dict(targets=None), dict(weight=None), dict(grad=None),
                                         dict(grad_ld=9), dict(grad=A + 2), dict(per_row=-1)]] + [
    (_grad, dict(per_row=16385), UNSUPPORTED)] + [
    (_embed, b, INVALID) for b in [dict(dtype=7), dict(table=None), dict(ids=None), dict(out=None),
                                   dict(ld=3), dict(out_ld=3), dict(n=-1), dict(V=-1), dict(D=-1),
                                   dict(n=1 << 31), dict(table=A + 2), dict(out=A + 1, dtype=2),
                                   dict(ids=A + 2)]] + [
    (_embed, dict(D=65537, ld=65537, out_ld=65537), UNSUPPORTED)] + [
    (_embed_grad, b, INVALID) for b in [dict(dtype=5), dict(grad_dtype=2), dict(grad_dtype=9),
                                        dict(dout=None), dict(ids=None), dict(grad=None),
                                        dict(dout_ld=3), dict(grad_ld=3), dict(n=-1), dict(V=-1),
                                        dict(ws=None), dict(ws=A + 64), dict(ws_bytes=16),
                                        dict(grad=A + 2), dict(dout=A + 1)]] + [
    (_embed_grad, dict(D=65537, dout_ld=65537, grad_ld=65537), UNSUPPORTED)])
def test_refusals(call, bad, status):
    assert call(**bad) == status
    name = {"_sample": "ml2_sample", "_logprob": "ml2_logprob", "_grad": "ml2_logprob_grad",
            "_embed": "ml2_embed", "_embed_grad": "ml2_embed_grad"}[call.__name__]
    assert ml2.lib().ml2_last_error().decode().startswith(name + ":")


def test_nothing_to_do_is_no_error():
    """Calls over nothing enqueue nothing (and need no GPU)."""
    assert _sample(rows=0, scores=None) == OK
    assert _sample(draws=0, u=None, idx=None, logprob=None) == OK
    assert _logprob(rows=0) == OK and _logprob(per_row=0, targets=None) == OK
    assert _grad(rows=0) == OK
    assert _embed(n=0, ids=None) == OK and _embed(D=0, ld=0, out_ld=0) == OK
    assert _embed_grad(V=0, grad=None) == OK


def test_workspace_queries():
    L, size = ml2.lib(), ctypes.c_size_t()
    for f in (L.ml2_sample_workspace_bytes, L.ml2_logprob_workspace_bytes):
        assert f(1000, 4, 2, ctypes.byref(size)) == OK and size.value >= 256
        assert f(0, 0, 0, ctypes.byref(size)) == OK
        assert f(1 << 24, 1, 16384, ctypes.byref(size)) == OK and size.value < 1 << 28
        assert f(-1, 4, 2, ctypes.byref(size)) == INVALID
        assert f(10, 4, 2, None) == INVALID
        assert f(10, 4, 16385, ctypes.byref(size)) == UNSUPPORTED
        assert f(10, 2097153, 2, ctypes.byref(size)) == UNSUPPORTED
    f = L.ml2_embed_grad_workspace_bytes
    assert f(32768, 131072, 1024, ctypes.byref(size)) == OK and size.value < 1 << 27
    assert f(0, 0, 0, ctypes.byref(size)) == OK
    assert f(10, -1, 4, ctypes.byref(size)) == INVALID
    assert f(10, 4, 4, None) == INVALID
    assert f(10, 4, 65537, ctypes.byref(size)) == UNSUPPORTED


def test_header_limits_match_binding():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "ml2.h")).read()
    for name in ("ML2_MAX_ROWS", "ML2_MAX_WIDTH"):
        m = re.search(rf"#define {name} (\d+)", text)
        assert m and int(m.group(1)) == getattr(ml2, name)
    for name in ("ML2_F32", "ML2_BF16", "ML2_F16"):
        assert re.search(rf"{name} = {getattr(ml2, name)}\b", text)


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="device"):
        ml2.ml2_sample(x, x, x, x, x)
    with pytest.raises(ValueError, match="device"):
        ml2.ml2_embed(x, x, x)
