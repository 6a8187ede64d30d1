"""ml2_layer_norm and ml2_layer_norm_grad against the formulas in 64 bits, within the tolerances
that tests/trainutil.py derives."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402
from tests import trainutil as t  # noqa: E402
from tests.trainutil import TYPES, wide  # noqa: E402

DEV = "cuda:0"
# around vectors of 4 and 8, groups of lanes, a wave, a workgroup, and the borders of each way
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 250, 256, 257, 511,
          512, 513, 771, 1000, 1023, 1024, 1025, 1500, 2047, 2048, 2049, 4096, 5003, 8191, 8192,
          8193, 16383, 16384, 16385, 20001, 32767, 32768, 32769, 50021, 65535, 65536]


def _rows(rng, rows, width, dtype, pad=0, kind="normal"):
    x = rng.standard_normal((rows, width + pad))
    if kind == "normal":
        x *= rng.uniform(0.1, 3.0, (rows, 1))
        x += rng.standard_normal((rows, 1))
    elif kind == "far":  # the mean is thousands of deviations away
        x += 10.0 ** rng.uniform(2, 4, (rows, 1))
    elif kind == "outlier":
        x[:, 0] *= 1000
    elif kind == "one":  # rows of one value
        x[:] = rng.standard_normal((rows, 1)) * 100
    elif kind == "small":
        x *= 1e-6
    return torch.from_numpy(x).to(dtype)


def _params(rng, width, dtype):
    return torch.from_numpy(1 + 0.3 * rng.standard_normal(width)).to(dtype), \
        torch.from_numpy(rng.standard_normal(width)).to(dtype)


def _forward(x, w, b, eps=1e-5, out=None, pad=0):
    """Checks a forward pass over x (a CPU tensor [rows][width + pad])."""
    rows, width = x.shape[0], x.shape[1] - pad
    xd = x.to(DEV)
    full = torch.full_like(xd, 4.0)
    mean, rstd = (torch.full((rows,), 7.0, device=DEV) for _ in range(2))
    wd, bd = (None if p is None else p.to(DEV) for p in (w, b))
    ml2.ml2_layer_norm(xd[:, :width], wd, bd, full[:, :width], mean, rstd, eps)
    torch.cuda.synchronize()
    xs, ws, bs = wide(x)[:, :width], wide(w), wide(b)
    y, m, r, xhat = t.layer_norm(xs, ws, bs, float(np.float32(eps)))
    tol, mtol, rtol = t.layer_norm_tolerance(xs, ws, xhat, y, r, x.dtype)
    assert t.close(wide(full)[:, :width], y, tol, x.dtype)
    assert np.all(np.abs(wide(mean) - m) <= mtol)
    assert np.all(np.abs(wide(rstd) - r) <= rtol)
    assert torch.all(full[:, width:] == 4.0)
    return xd, wd, mean, rstd


def _backward(rng, x, w, eps, pad, grad_dtype, xd, wd, mean, rstd, bias=True):
    rows, width = x.shape[0], x.shape[1] - pad
    dout = _rows(rng, rows, width, x.dtype, pad)
    dd = dout.to(DEV)
    dx = torch.full_like(xd, 4.0)
    dw = torch.full((width,), 9.0, dtype=grad_dtype, device=DEV)
    db = torch.full((width,), 9.0, dtype=grad_dtype, device=DEV) if bias else None
    need = ml2.ml2_layer_norm_grad_workspace_bytes(rows, width)
    ws = torch.full((max(256, need),), 255, dtype=torch.uint8, device=DEV)
    ml2.ml2_layer_norm_grad(xd[:, :width], dd[:, :width], wd, mean, rstd, ws, dx[:, :width], dw, db)
    torch.cuda.synchronize()
    args = wide(x)[:, :width], wide(dout)[:, :width], wide(w), wide(rstd)
    gx, gw, gb, _ = t.layer_norm_grad(*args)
    tx, tw, tb = t.layer_norm_grad_tolerance(*args, gx, gw, gb, x.dtype, grad_dtype)
    assert t.close(wide(dx)[:, :width], gx, tx, x.dtype)
    assert t.close(wide(dw), gw, tw, grad_dtype)
    if bias:
        assert t.close(wide(db), gb, tb, grad_dtype)
    assert torch.all(dx[:, width:] == 4.0)


def _both(dtype, rows, width, pad=0, kind="normal", params=torch.float32, grads=None,
          weight=True, bias=True, eps=1e-5):
    print(f"[layer_norm] {dtype} {rows} x {width} + {pad} {kind}", flush=True)
    rng = np.random.default_rng(rows * 70001 + width + pad)
    x = _rows(rng, rows, width, dtype, pad, kind)
    w, b = _params(rng, width, params)
    w, b = (w if weight else None), (b if bias else None)
    xd, wd, mean, rstd = _forward(x, w, b, eps, pad=pad)
    _backward(rng, x, w, eps, pad, grads or params, xd, wd, mean, rstd, bias)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(dtype, width):
    _both(dtype, 7 if width < 20000 else 3, width, params=dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [1, 5, 63, 64, 130, 771, 1030, 5003, 20003])
@pytest.mark.parametrize("pad", [1, 8])
def test_strides(dtype, width, pad):
    _both(dtype, 37, width, pad, grads=dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 64), (1, 65536), (2, 3), (64, 8), (255, 8),
                                        (257, 17), (1000, 128), (4097, 33), (5000, 512),
                                        (3001, 771), (20000, 5), (300, 2050), (1100, 1040),
                                        (270, 16384), (512, 8200), (513, 8200),
                                        (600, 16384), (515, 20001), (513, 24576), (100, 16390), (70000, 2), (17, 512), (65, 512),
                                        (32, 1024), (33, 1024), (4, 4096), (5, 4096)])
def test_rows(dtype, rows, width):
    _both(dtype, rows, width)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [
    (64, 8193), (65, 8193), (320, 8193), (321, 8193), (64, 20001), (65, 20001),  # read twice
    (2, 8192), (3, 8192), (8, 4096), (9, 4096), (1, 12288), (1, 12289), (2, 12288),  # launches
    (2032, 1024), (2033, 1001), (4080, 600), (4081, 600), (16257, 60), (20000, 9),  # waves
    (12400, 100), (9000, 200), (4100, 257)])
def test_rows_at_the_gradients_borders(dtype, rows, width):
    _both(dtype, rows, width)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["far", "outlier", "one", "small"])
@pytest.mark.parametrize("width", [6, 64, 771, 3000, 17000])
def test_values(dtype, kind, width):
    if kind == "far" and dtype is not torch.float32:
        kind = "one"  # 8 or 11 bits leave one value of such rows
    _both(dtype, 11, width, kind=kind, eps=1e-12 if kind == "small" else 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [40, 1024, 2100, 16500])
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_parameters(dtype, width, weight, bias):
    _both(dtype, 9, width, weight=weight, bias=bias, grads=dtype)


@pytest.mark.parametrize("width", [8, 700, 1500, 17001])
def test_nan_and_infinity_stay_in_their_rows(width):
    rng = np.random.default_rng(width)
    x = _rows(rng, 6, width, torch.float32)
    clean = x.clone()
    x[1, width // 2], x[3, width - 1], x[4, 0] = np.nan, np.inf, -np.inf
    w, b = (p.to(DEV) for p in _params(rng, width, torch.float32))
    dout = _rows(rng, 6, width, torch.float32).to(DEV)
    got = []
    for rows in (x, clean):
        ln, grad = ml2.LayerNorm(6, width, x.dtype), ml2.LayerNormGrad(6, width, x.dtype)
        out, mean, rstd = ln.run(rows.to(DEV), w, b)
        dx, dw, db = grad.run(rows.to(DEV), dout, w, mean, rstd)
        got.append([v.cpu() for v in (out, dx, dw, db)])
    bad = torch.tensor([False, True, False, True, True, False])
    for have, want in zip(got[0][:2], got[1][:2]):
        assert torch.isnan(have[bad]).all() and torch.equal(have[~bad], want[~bad])
    assert torch.isnan(got[0][2]).all()  # every column's sum has such a row
    assert torch.equal(got[0][3], got[1][3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(50, 24), (50, 1000), (50, 3001), (50, 18000), (520, 8300),
                                        (515, 17001), (700, 24)])
def test_in_place(dtype, rows, width):
    """The output in the rows' memory, the rows' gradient in x's and in dout's."""
    rng = np.random.default_rng(width)
    x, dout = (_rows(rng, rows, width, dtype, 3).to(DEV)[:, :width] for _ in range(2))
    w, b = (p.to(DEV) for p in _params(rng, width, torch.float32))
    ln = ml2.LayerNorm(rows, width, dtype)
    out, mean, rstd = ln.run(x, w, b)
    grad = ml2.LayerNormGrad(rows, width, dtype, torch.float32)
    dx, dw, db = grad.run(x, dout, w, mean, rstd)
    for into in ("x", "dout"):
        a = torch.empty(rows, width + 3, dtype=dtype, device=DEV)[:, :width]
        d = torch.empty(rows, width + 5, dtype=dtype, device=DEV)[:, :width]
        a.copy_(x)
        d.copy_(dout)
        to = a if into == "x" else d
        gw, gb = torch.empty_like(dw), torch.empty_like(db)
        ml2.ml2_layer_norm_grad(a, d, w, mean, rstd, grad.ws, to, gw, gb)
        torch.cuda.synchronize()
        assert torch.equal(to, dx) and torch.equal(gw, dw) and torch.equal(gb, db)
    y = x.clone()
    ml2.ml2_layer_norm(y, w, b, y)
    torch.cuda.synchronize()
    assert torch.equal(y, out)


@pytest.mark.parametrize("width", [24, 1000, 3001, 18000])
def test_parts_alone(width):
    """Each gradient alone has the bits that it has beside the others."""
    rng = np.random.default_rng(width)
    x, dout = (_rows(rng, 40, width, torch.bfloat16).to(DEV) for _ in range(2))
    w, b = (p.to(DEV) for p in _params(rng, width, torch.float32))
    _, mean, rstd = ml2.LayerNorm(40, width, x.dtype).run(x, w, b)
    grad = ml2.LayerNormGrad(40, width, x.dtype)
    all_of = [v.clone() for v in grad.run(x, dout, w, mean, rstd)]
    for i in range(3):
        for v in (grad.dx, grad.dweight, grad.dbias):
            v.fill_(3.0)
        outs = [v if j == i else None for j, v in enumerate((grad.dx, grad.dweight, grad.dbias))]
        ml2.ml2_layer_norm_grad(x, dout, w, mean, rstd, grad.ws, *outs)
        torch.cuda.synchronize()
        assert torch.equal(outs[i], all_of[i])


def test_nothing_to_do():
    for rows, width in ((0, 5), (3, 0), (0, 0), (0, 20000)):
        x = torch.empty(rows, width, device=DEV)
        out, mean, rstd = ml2.LayerNorm(rows, width, x.dtype).run(x)
        grad = ml2.LayerNormGrad(rows, width, x.dtype)
        grad.dweight.fill_(2.0)
        grad.dbias.fill_(2.0)
        _, dw, db = grad.run(x, torch.empty_like(x), None, mean, rstd)
        torch.cuda.synchronize()
        assert torch.all(dw == 0) and torch.all(db == 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_far_apart(dtype):
    """Offsets beyond 2^31 elements."""
    width, ld = 40, (1 << 30) + 40
    rng = np.random.default_rng(1)
    rows = _rows(rng, 3, width, dtype)
    buf = torch.empty(2 * ld + width, dtype=dtype, device=DEV)
    x = torch.as_strided(buf, (3, width), (ld, 1))
    x.copy_(rows)
    w, b = (p.to(DEV) for p in _params(rng, width, dtype))
    dout = _rows(rng, 3, width, dtype).to(DEV)
    out, mean, rstd = ml2.LayerNorm(3, width, dtype).run(x.clone(), w, b)
    dx, dw, db = ml2.LayerNormGrad(3, width, dtype).run(x.clone(), dout, w, mean, rstd)
    grad = ml2.LayerNormGrad(3, width, dtype)
    ml2.ml2_layer_norm_grad(x, dout, w, mean, rstd, grad.ws, x, grad.dweight, grad.dbias)
    torch.cuda.synchronize()
    assert torch.equal(x, dx) and torch.equal(grad.dweight, dw) and torch.equal(grad.dbias, db)
    x.copy_(rows)
    ml2.ml2_layer_norm(x, w, b, x)
    torch.cuda.synchronize()
    assert torch.equal(x, out)


@pytest.mark.parametrize("rows,width", [(96, 128), (2000, 700), (64, 20000)])
def test_streams_graph_and_repeats(rows, width):
    """The same bits on another stream, on every replay of a captured graph with eager work
    between the replays, and in every run."""
    rng = np.random.default_rng(rows)
    x, dout = (_rows(rng, rows, width, torch.bfloat16).to(DEV) for _ in range(2))
    w, b = (p.to(DEV) for p in _params(rng, width, torch.float32))
    ln, grad = ml2.LayerNorm(rows, width, x.dtype), ml2.LayerNormGrad(rows, width, x.dtype)

    def step(stream=None):
        out, mean, rstd = ln.run(x, w, b, stream=stream)
        return (out, mean, rstd, *grad.run(x, dout, w, mean, rstd, stream=stream))

    want = [v.clone() for v in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for v in step(side):
        pass
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(step(), want))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for turn in range(4):
        for v in got:
            v.fill_(5.0)
        x2 = x.clone()
        if turn % 2:
            x.mul_(2.0)
        want = [v.clone() for v in (_eager(x, dout, w, b))]
        for v in got:
            v.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        x.copy_(x2)


def _eager(x, dout, w, b):
    out, mean, rstd = ml2.LayerNorm(*x.shape, x.dtype).run(x, w, b)
    return (out, mean, rstd, *ml2.LayerNormGrad(*x.shape, x.dtype).run(x, dout, w, mean, rstd))


@pytest.mark.parametrize("width", [2, 100, 1000, 5000, 20000, 50021])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_whose_sum_passes_float32(width, dtype):
    """2^127 and another number of 2^127 are 2^128: such a row is NaN, the one beside it is not."""
    x = torch.zeros(3, width, device=DEV, dtype=dtype)
    x[0, :2] = 2.0 ** 127
    x[1, :1] = 2.0 ** 60
    x[2, 0], x[2, 1] = 2.0 ** 64, -2.0 ** 64  # squares that pass it: an rstd of 0
    out, mean, rstd = ml2.LayerNorm(3, width, dtype).run(x)
    assert out[0].isnan().all() and mean[0].isnan() and rstd[0].isnan()
    assert out[1].isfinite().all() and mean[1].isfinite() and rstd[1] > 0
    assert (out[2] == 0).all() and mean[2] == 0 and rstd[2] == 0


def test_tensors_of_another_device_are_refused(monkeypatch):
    """A call goes to the current device's stream: tensors of another one (here: seen so) raise."""
    x = torch.zeros(4, 8, device=DEV)
    ln, grad = ml2.LayerNorm(4, 8, x.dtype), ml2.LayerNormGrad(4, 8, x.dtype)
    out, mean, rstd = ln.run(x)
    norm, adam = ml2.GradNorm([x]), ml2.AdamW([x], [x.clone()])
    monkeypatch.setattr(ml2._t(), "current", lambda: 1)
    for call in (lambda: ln.run(x), lambda: grad.run(x, x, None, mean, rstd), norm.run,
                 lambda: adam.run(1e-3, 1), lambda: ml2.ml2_layer_norm(x, None, None, out),
                 lambda: ml2.ml2_layer_norm_grad(x, x, None, mean, rstd, grad.ws, grad.dx),
                 lambda: ml2.ml2_grad_norm([x], norm.norm, norm.factor, norm.ws)):
        with pytest.raises(ValueError, match="current"):
            call()


def test_objects_refuse_other_rows():
    x = torch.zeros(4, 8, device=DEV)
    ln, grad = ml2.LayerNorm(4, 8, x.dtype), ml2.LayerNormGrad(4, 8, x.dtype)
    _, mean, rstd = ln.run(x)
    w = torch.ones(8, device=DEV)
    for call in (lambda: ln.run(x[:3]), lambda: ln.run(x[:, :7]), lambda: ln.run(x.half()),
                 lambda: ln.run(x, w[:7]), lambda: ln.run(x, w.half(), w),
                 lambda: grad.run(x, x[:3], w, mean, rstd), lambda: grad.run(x, x.half(), w, mean, rstd),
                 lambda: grad.run(x, x, w.half(), mean, rstd),
                 lambda: grad.run(x, x, w, mean[:3], rstd), lambda: ln.run(x.t().contiguous().t())):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width", [(9, 24), (70, 1000), (9, 17000)])
def test_arrays_between_the_rows(dtype, rows, width):
    """Parameters, statistics, sums and the workspace in the columns behind the rows of one buffer:
    the same bits as in memory of their own."""
    print(f"[layer_norm] between rows: {dtype} {rows} x {width}", flush=True)
    rng = np.random.default_rng(rows + width)
    x, dout = (_rows(rng, rows, width, dtype).to(DEV) for _ in range(2))
    w, b = (p.to(DEV) for p in _params(rng, width, torch.float32))
    need = ml2.ml2_layer_norm_grad_workspace_bytes(rows, width)
    span = -(-width * 4 // 256) * 256  # bytes of a row and of each array in a row's gap
    pitch = 2 * span + -(-need // 256) * 256
    whole = torch.full((5 * rows * pitch,), 77, dtype=torch.uint8, device=DEV)
    free = torch.ones(5 * rows, pitch, dtype=torch.bool, device=DEV)

    def rows_of(i):  # the rows i, i + 5, ... of the buffer
        view = whole.view(dtype).view(5 * rows, -1)[i::5, :width]
        free[i::5, :width * dtype.itemsize] = False
        return view

    def behind(row, n):
        at = row * pitch + span
        free.view(-1)[at: at + 4 * n] = False
        return whole[at: at + 4 * n].view(torch.float32)

    xs, ds, out, dx = (rows_of(i) for i in range(4))
    ws, bs, dw, db = (behind(row, width) for row in (0, 1, 2, 3))
    mean, rstd = (behind(row, rows) for row in (4, 5))
    at = 7 * pitch + 2 * span
    space = whole[at: at + max(need, 1)]
    free.view(-1)[at: at + max(need, 1)] = False
    for to, v in ((xs, x), (ds, dout), (ws, w), (bs, b)):
        to.copy_(v)
    ml2.ml2_layer_norm(xs, ws, bs, out, mean, rstd)
    ml2.ml2_layer_norm_grad(xs, ds, ws, mean, rstd, space, dx, dw, db)
    ln, grad = ml2.LayerNorm(rows, width, dtype), ml2.LayerNormGrad(rows, width, dtype, torch.float32)
    want = ln.run(x, w, b)
    want += grad.run(x, dout, w, want[1], want[2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, v) for a, v in zip((out, mean, rstd, dx, dw, db), want))
    assert torch.equal(xs, x) and torch.equal(ds, dout) and torch.equal(ws, w)
    assert torch.all(whole[free.view(-1)] == 77)
    inside = whole[2 * pitch: 2 * pitch + 4 * rows].view(torch.float32)  # out's first row
    with pytest.raises(ml2.Ml2Error, match="shares memory"):
        ml2.ml2_layer_norm(xs, ws, bs, out, inside, rstd)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("params", ["float32", "rows"])
@pytest.mark.parametrize("rows,width", [(600, 50021), (1700, 33000), (1700, 20001), (4500, 9000),
                                        (700, 65536)])
def test_more_rows_than_workgroups(dtype, params, rows, width):
    """A wide row has the same bits whatever other rows a call has: as one of so many that
    workgroups take several, or have one each, and among 100.  Some of them, on both sides of
    where workgroups begin their second row, are held against 64 bits too."""
    print(f"[layer_norm] many rows: {dtype} {params} {rows} x {width}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(rows + width)
    x = torch.empty(rows, width, dtype=dtype, device=DEV)
    for at in range(0, rows, 100):
        x[at: at + 100] = torch.randn(min(100, rows - at), width, generator=g, device=DEV) * 1.7 + 0.4
    w, b = (p.to(DEV) for p in _params(np.random.default_rng(width), width,
                                       torch.float32 if params == "float32" else dtype))
    out, mean, rstd = ml2.LayerNorm(rows, width, dtype).run(x, w, b)
    for at in range(0, rows, 100):
        few = ml2.LayerNorm(len(x[at: at + 100]), width, dtype).run(x[at: at + 100], w, b)
        for have, want in zip((out, mean, rstd), few):
            assert torch.equal(have[at: at + 100], want)
    some = [r for r in (0, 255, 256, 511, 512, 1023, 1535, 1536) if r < rows - 1] + [rows - 1]
    y, m, r, xhat = t.layer_norm(wide(x[some]), wide(w), wide(b), float(np.float32(1e-5)))
    tol, mtol, rtol = t.layer_norm_tolerance(wide(x[some]), wide(w), xhat, y, r, dtype)
    assert t.close(wide(out[some]), y, tol, dtype)
    assert np.all(np.abs(wide(mean[some]) - m) <= mtol)
    assert np.all(np.abs(wide(rstd[some]) - r) <= rtol)
