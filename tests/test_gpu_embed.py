"""ml2_embed and ml2_embed_grad against the formula in 64 bits.

The lookup is one float32 product rounded once: it must equal that bit for
bit.  A gradient's sum of k terms is within k 2^-24 of the sum of their sizes,
plus the rounding to its type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402
from tests import drawutil  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _ids(rng, n, V, skew):
    if skew:
        ids = np.minimum(V - 1, np.exp(rng.random(n) * np.log(V + 1.0)).astype(np.int64) - 1)
    else:
        ids = rng.integers(0, V, n)
    ids = ids.astype(np.int32)
    ids[rng.random(n) < 0.05] = -1
    ids[rng.random(n) < 0.02] = V
    return ids


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,D", [(0, 5, 8), (1, 1, 1), (7, 3, 2), (65, 100, 7), (130, 50, 64),
                                   (1000, 4096, 128), (33, 9, 1023), (20000, 81, 1),
                                   (3, 4, 65536), (5, 0, 16)])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_lookup(dtype, n, V, D, pad):
    rng = np.random.default_rng(n + V + D)
    table = torch.from_numpy(rng.standard_normal((V, D + pad)).astype(np.float32)).to(dtype)
    ids = _ids(rng, n, max(V, 1), False)
    out = torch.full((n, D + pad), 4.0, dtype=dtype, device=DEV)
    ml2.ml2_embed(table.to(DEV)[:, :D], torch.from_numpy(ids).to(DEV), out[:, :D], 1.7)
    torch.cuda.synchronize()
    ok = torch.from_numpy((ids >= 0) & (ids < V))
    want = torch.zeros(n, D, dtype=dtype)
    if V:
        rows = (table[:, :D].float() * torch.tensor(1.7)).to(dtype)
        want[ok] = rows[torch.from_numpy(ids)[ok].long()]
    assert torch.equal(out[:, :D].cpu(), want)
    assert torch.all(out[:, D:] == 4.0)
    ref = drawutil.embed(drawutil.as_float(table)[:, :D], ids, 1.7)
    got = drawutil.as_float(out[:, :D])
    assert np.all(np.abs(got - ref) <= (ROUND[dtype] + 2.0 ** -23) * np.abs(ref) + 1e-7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n,V,D,skew", [
    (0, 7, 5, False), (1, 1, 1, False), (1, 1000, 3, False), (31, 4, 9, True), (64, 1, 1, False),
    (500, 2, 1, True), (2000, 81, 1, False), (4097, 300, 40, True), (3000, 5000, 129, False),
    (9000, 17, 256, True), (1025, 600, 513, True), (100, 70000, 16, True), (70001, 81, 2, True),
    (300000, 7, 1, True), (270000, 100000, 3, False), (50, 9, 4099, True), (513, 200000, 1, False),
    (8192, 3000, 2, True), (8193, 70000, 5, False), (600000, 70000, 2, True)])
def test_gradient(dtype, wide, n, V, D, skew):
    print(f"[embed_grad] {dtype} wide={wide} n={n} V={V} D={D}", flush=True)
    rng = np.random.default_rng(n + V + D)
    for pad in (0, 3):
        dout = torch.from_numpy(rng.standard_normal((n, D + pad)).astype(np.float32)).to(dtype)
        ids = _ids(rng, n, V, skew)
        out = torch.float32 if wide else dtype
        grad = torch.full((V, D + pad), 4.0, dtype=out, device=DEV)
        ws = torch.full((max(256, ml2.ml2_embed_grad_workspace_bytes(n, V, D)),), 255,
                        dtype=torch.uint8, device=DEV)
        ml2.ml2_embed_grad(dout.to(DEV)[:, :D], torch.from_numpy(ids).to(DEV), grad[:, :D], ws, 0.3)
        torch.cuda.synchronize()
        d = drawutil.as_float(dout)[:, :D]
        want = drawutil.embed_grad(d, ids, V, np.float64(np.float32(0.3)))
        size = drawutil.embed_grad(np.abs(d), ids, V, 0.3)
        terms = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
        tol = (terms + 2) * 2.0 ** -24 * size + ROUND[out] * np.abs(want) + 1e-7
        got = drawutil.as_float(grad[:, :D])
        assert np.all(np.abs(got - want) <= tol)
        assert torch.all(grad[:, D:] == 4.0)


def test_gradient_is_the_lookups_transpose():
    """<dout, lookup(table + d) - lookup(table)> = <d, gradient>, in whole
    numbers small enough that every sum is exact."""
    rng = np.random.default_rng(8)
    n, V, D = 700, 90, 33
    table = torch.from_numpy(rng.integers(-8, 9, (V, D)).astype(np.float32)).to(DEV)
    d = torch.from_numpy(rng.integers(-8, 9, (V, D)).astype(np.float32)).to(DEV)
    dout = torch.from_numpy(rng.integers(-8, 9, (n, D)).astype(np.float32)).to(DEV)
    ids = torch.from_numpy(_ids(rng, n, V, True)).to(DEV)
    e = ml2.Embedding(n, D, torch.float32)
    a = e.run(table + d, ids, 2.0).clone()
    b = e.run(table, ids, 2.0)
    g = ml2.EmbeddingGrad(n, V, D, torch.float32).run(dout, ids, 2.0)
    assert float(((a - b).double() * dout.double()).sum()) == float((d.double() * g.double()).sum())


def test_same_bits_every_run_and_in_a_graph():
    rng = np.random.default_rng(10)
    for n, V, D in ((300000, 50, 2), (5000, 700, 130)):
        dout = torch.randn(n, D, device=DEV)
        ids = torch.from_numpy(_ids(rng, n, V, True)).to(DEV)
        f = ml2.EmbeddingGrad(n, V, D, torch.float32)
        want = f.run(dout, ids).clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        f.run(dout, ids, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(want, f.grad)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f.run(dout, ids)
        for _ in range(4):
            f.grad.fill_(9.0)
            f.ws.fill_(255)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(want, f.grad)
            dout.mul_(0.9)
            want = f.run(dout, ids).clone()
