"""The operators of a training step together, as examples/policy_explorer.py's network uses them
beside the lookups and the loss: gradients against 64 bits and against differences, steps eager
and captured."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
from examples import policy_explorer  # noqa: E402
from paper_2411_10764_amd import ml2  # noqa: E402

N, FAMILIES, WIDTH, DRAWS = 300, 12, 24, 16


def _problem(seed=3):
    g = torch.Generator().manual_seed(seed)
    family = torch.randint(FAMILIES, (N,), generator=g, dtype=torch.int32).to("cuda")
    targets = torch.randint(N, (1, DRAWS), generator=g, dtype=torch.int32).to("cuda")
    weight = torch.randn(1, DRAWS, generator=g).to("cuda")
    return family, targets, weight


def _network(bits=32):
    net = policy_explorer.Network(N, FAMILIES, WIDTH, 0.01, seed=7, state_bits=bits)
    net.weight += 0.3 * torch.sin(torch.arange(WIDTH, device="cuda"))
    net.bias += 0.1
    return net


def _loss(params, family, targets, weight):
    """-sum of weighted log-probabilities, in 64 bits on the CPU, by torch's autograd"""
    table, w, b, head = params
    x = table[family.cpu().long()]
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    y = ((x - mean) / torch.sqrt(var + 1e-5) * w + b) @ head
    logp = torch.log_softmax(y, 0)
    return -(logp[targets[0].cpu().long()] * weight[0].cpu().double()).sum()


def _gradients(net, likelihood, family, targets, weight):
    logits = net.forward(family).view(1, N)
    _, d = likelihood.run_grad(logits, targets, weight)
    net.backward(family, -d[0])


def _sizes(params, family, targets, weight):
    """Of every gradient's element, the sum of the sizes of the terms that it is the sum of: the
    gradient to a logit has those of its probability times all weights and of the weights of its
    draws (they cancel in the sum over the logits, so the bias's gradient is 0), and goes on
    through products with what is given here."""
    table, w, b, head = (np.abs(p.detach().numpy()) for p in params)
    rows = family.cpu().numpy()
    x = params[0].detach().numpy()
    xhat = x - x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(np.square(xhat).mean(1) + 1e-5)
    xhat = np.abs(xhat * rstd[:, None])[rows]
    with torch.no_grad():
        z = params[0][rows.astype(np.int64)]
        m = z.mean(1, keepdim=True)
        logits = ((z - m) / torch.sqrt((z - m).square().mean(1, keepdim=True) + 1e-5) * params[1]
                  + params[2]) @ params[3]
        prob = torch.softmax(logits, 0).numpy()
    v = np.abs(weight[0].cpu().numpy().astype(np.float64))
    dy = prob * v.sum()
    np.add.at(dy, targets[0].cpu().numpy(), v)
    g = dy[:, None] * head * w
    dx = rstd[rows][:, None] * (g + g.mean(1, keepdims=True)
                                + xhat * (g * xhat).mean(1, keepdims=True))
    dtable = np.zeros_like(table)
    np.add.at(dtable, rows, dx)
    return (dtable, (dy[:, None] * head * xhat).sum(0), (dy[:, None] * head).sum(0),
            (dy[:, None] * (xhat * w + b)).sum(0))


def test_gradients_are_those_of_the_loss():
    """A term of a gradient goes through five operators (lookup, norm, logits, loss, and the norm's
    or the table's gradient), each of which rounds it at most 600 times, additions to at most 300
    others among them: 3,000 roundings of 2^-24, of the sizes above.  Differences of the 64-bit
    loss agree with its autograd."""
    net, (family, targets, weight) = _network(), _problem()
    likelihood = ml2.LogProb(1, N, DRAWS, grad_dtype=torch.float32)
    _gradients(net, likelihood, family, targets, weight)
    torch.cuda.synchronize()
    params = [p.detach().cpu().double().requires_grad_() for p in net.adam.params]
    loss = _loss(params, family, targets, weight)
    loss.backward()
    rng = np.random.default_rng(1)
    for p, have, size in zip(params, net.adam.grads, _sizes(params, family, targets, weight)):
        want, got = p.grad.numpy(), have.cpu().double().numpy()
        assert np.all(np.abs(got - want) <= 3000 * 2.0 ** -24 * size)
        v, h = torch.from_numpy(rng.standard_normal(p.shape)), 1e-6
        with torch.no_grad():
            p += h * v
            up = _loss(params, family, targets, weight)
            p -= 2 * h * v
            down = _loss(params, family, targets, weight)
            p += h * v
        slope = float(up - down) / (2 * h)
        assert abs(slope - float((torch.from_numpy(want) * v).sum())) < 1e-6 * (1 + abs(slope))


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_captured_and_eager(bits):
    """The whole step in one graph: every replay has the bits of the eager step, with eager work and
    a synchronization between replays; a step whose gradients are not finite is left out."""
    family, targets, weight = _problem()
    nets = [_network(bits) for _ in range(2)]
    losses = [ml2.LogProb(1, N, DRAWS, grad_dtype=torch.float32) for _ in range(2)]

    def step(i):
        _gradients(nets[i], losses[i], family, targets, weight)
        nets[i].step()

    for i in (0, 1):
        step(i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for turn in range(6):
        weight.copy_(torch.randn(1, DRAWS, device="cuda"))
        if turn == 3:
            weight[0, 2] = float("nan")
        before = [p.clone() for p in nets[1].adam.params]
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        for a, b in zip(nets[0].adam.params, nets[1].adam.params):
            assert torch.equal(a, b)
        for a, b in zip(nets[0].adam.m + nets[0].adam.v, nets[1].adam.m + nets[1].adam.v):
            assert torch.equal(a, b)
        same = all(torch.equal(a, b) for a, b in zip(before, nets[1].adam.params))
        assert same == (turn == 3)
        assert int(nets[0].count) == int(nets[1].count) == turn + (2 if turn < 3 else 1)


def test_the_example_runs_and_repeats():
    a = policy_explorer.run(rounds=12, width=16)
    assert len(a) == 12 and all(np.isfinite(a))
    assert policy_explorer.run(rounds=12, width=16) == a
