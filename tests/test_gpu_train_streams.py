"""The operators of a training step on a stream that is not the current one: what they read is
still being made there when they are called, so a call that went to another stream would find the
old values, and what they write is looked at after that stream alone."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402

DEV = "cuda:0"


def _after_work(side, pairs):
    """Queues some milliseconds of products on the stream and then copies, as (to, from)."""
    a = torch.full((4096, 4096), 1.0 / 4096, device=DEV)
    b = torch.empty_like(a)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(12):
            torch.mm(a, a, out=b)
        for to, new in pairs:
            to.copy_(new)
    return a, b  # kept until the stream is through


def _check(side, inputs, call, outputs):
    """`inputs`: (tensor, its new values); call(stream); outputs(): what it has written."""
    old = [x.clone() for x, _ in inputs]
    for x, new in inputs:
        x.copy_(new)
    call(None)
    torch.cuda.synchronize()
    want = [x.clone() for x in outputs()]
    for stream in (side, side.cuda_stream):
        for _ in range(5):
            for (x, _), v in zip(inputs, old):
                x.copy_(v)
            for x in outputs():
                x.fill_(5)
            kept = _after_work(side, inputs)
            call(stream)
            running = not side.query()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outputs(), want))
            del kept
            if running:  # the products still were when the call returned; else once more
                break
        assert running


@pytest.mark.parametrize("rows,width", [(96, 128), (2000, 700), (100, 20000)])
def test_layer_norm(rows, width):
    side = torch.cuda.Stream()
    x, dout, new_x, new_dout = (torch.randn(rows, width, device=DEV).bfloat16() for _ in range(4))
    w, b = torch.randn(width, device=DEV), torch.randn(width, device=DEV)
    ln, grad = ml2.LayerNorm(rows, width, x.dtype), ml2.LayerNormGrad(rows, width, x.dtype)

    def call(stream):
        _, mean, rstd = ln.run(x, w, b, stream=stream)
        grad.run(x, dout, w, mean, rstd, stream=stream)

    _check(side, [(x, new_x), (dout, new_dout)], call,
           lambda: (ln.out, ln.mean, ln.rstd, grad.dx, grad.dweight, grad.dbias))

    def raw(stream):
        ml2.ml2_layer_norm(x, w, b, ln.out, ln.mean, ln.rstd, stream=stream)
        ml2.ml2_layer_norm_grad(x, dout, w, ln.mean, ln.rstd, grad.ws, grad.dx, grad.dweight,
                                grad.dbias, stream=stream)

    _check(side, [(x, new_x), (dout, new_dout)], raw,
           lambda: (ln.out, ln.mean, ln.rstd, grad.dx, grad.dweight, grad.dbias))


@pytest.mark.parametrize("sizes", [[50], [300000, 7]])
def test_norm(sizes):
    side = torch.cuda.Stream()
    grads, new = ([torch.randn(n, device=DEV) for n in sizes] for _ in range(2))
    norm = ml2.GradNorm(grads, 0.5)
    both = list(zip(grads, new))
    _check(side, both, lambda stream: norm.run(stream=stream), lambda: (norm.norm, norm.factor))
    _check(side, both,
           lambda stream: ml2.ml2_grad_norm(grads, norm.norm, norm.factor, norm.ws, 0.5,
                                            stream=stream), lambda: (norm.norm, norm.factor))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    side = torch.cuda.Stream()
    sizes = [3000, 512]
    params, grads, new = ([torch.randn(n, device=DEV) for n in sizes] for _ in range(3))
    out = [[torch.empty_like(p) for p in params],
           *([ml2.adamw_state(n, bits) for n in sizes] for _ in range(2))]
    plan = ml2.AdamW(params, grads, bits, out=out)
    rate, new_rate = torch.full((1,), 1.0, device=DEV), torch.full((1,), 2.0 ** -10, device=DEV)
    count, new_count = (torch.full((1,), n, dtype=torch.int32, device=DEV) for n in (90, 2))

    def written():  # without the bytes behind an 8-bit state's elements
        if bits == 32:
            return [x for xs in out for x in xs]
        return out[0] + [v.view(torch.uint8) for xs in out[1:] for x, n in zip(xs, sizes)
                         for v in ml2.adamw_state_parts(x, n)]

    _check(side, [*zip(grads, new), (rate, new_rate), (count, new_count)],
           lambda stream: plan.run(rate, count, stream=stream), written)
