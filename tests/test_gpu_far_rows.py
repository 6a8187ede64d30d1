"""Rows so far apart that an element's place passes 2^31 elements and 2^32 bytes:
every operator gives the bits that it gives on the same rows side by side."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402

DEV = "cuda:0"
FAR = (1 << 31) + 24  # elements from one row to the next


def _far(x, fill=None):
    """x's rows FAR elements apart (the memory between them is not touched)."""
    rows, n = x.shape
    out = torch.empty((rows - 1) * FAR + n, dtype=x.dtype, device=DEV).as_strided((rows, n), (FAR, 1))
    if fill is None:
        out.copy_(x)
    else:
        out.fill_(fill)
    return out


@pytest.fixture(autouse=True)
def _release():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1000, 20011, 70001, 300007])
def test_rows_of_scores(dtype, n):
    print(f"[far rows] scores {dtype} {n}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    rows = 2
    x = (torch.randn(rows, n, generator=g, device=DEV) * 2).to(dtype)
    valid = (torch.rand(rows, n, generator=g, device=DEV) < 0.6).to(torch.uint8)
    k = torch.full((rows,), 200, dtype=torch.int32, device=DEV)
    p = torch.full((rows,), 0.9, device=DEV)
    targets = torch.randint(n, (rows, 5), generator=g, device=DEV, dtype=torch.int32)
    weight = torch.randn(rows, 5, generator=g, device=DEV)
    fx, fv = _far(x), _far(valid)
    for draws in (1, 40):
        u = torch.rand(rows, draws, generator=g, device=DEV)
        got = [[t.clone() for t in ml2.Sampler(rows, n, draws).run(s, u, v, None, k, p)]
               for s, v in ((x, valid), (fx, fv))]
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    f = ml2.LogProb(rows, n, 5, grad_dtype=dtype)
    want = [t.clone() for t in f.run_grad(x, targets, weight, valid)]
    fg = _far(x, 3.0)
    f.logprob.fill_(7.0)
    ml2.ml2_logprob_grad(fx, targets, weight, fg, f.ws, f.logprob, fv)
    assert torch.equal(f.logprob, want[0]) and torch.equal(fg, want[1])
    f.logprob.fill_(7.0)
    assert torch.equal(f.run(fx, targets, fv), want[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width", [3, 200])
def test_tables(dtype, width):
    print(f"[far rows] table {dtype} {width}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(width)
    table = torch.randn(3, width, generator=g, device=DEV).to(dtype)
    ids = torch.tensor([2, 0, 2, -1], dtype=torch.int32, device=DEV)
    want = ml2.Embedding(4, width, dtype).run(table, ids, 0.7).clone()
    out = _far(want, 3.0)
    ml2.ml2_embed(_far(table), ids, out, 0.7)
    assert torch.equal(out, want)
    del out
    dout = torch.randn(4, width, generator=g, device=DEV).to(dtype)
    f = ml2.EmbeddingGrad(4, 3, width, torch.float32)
    want = f.run(dout, ids, 0.7).clone()
    grad = _far(want, 3.0)
    ml2.ml2_embed_grad(_far(dout), ids, grad, f.ws, 0.7)
    assert torch.equal(grad, want)
