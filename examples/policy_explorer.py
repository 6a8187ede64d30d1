"""An explorer that learns while it tunes: one learned number per pair of knob
values is added to the performance model's scores, candidates are drawn from
the softmax of the sum instead of taken greedily, and what was measured moves
the numbers by the gradient of its log-likelihood.

    python examples/policy_explorer.py [--rounds N] [--draws D] [--width W]

A round is
  1. the validity mask and the performance scores of the pool   ml2_score
  2. every candidate's learned number                           ml2_embed
  3. draws from the masked softmax of their sum                 ml2_sample
  4. the drawn candidates are measured (here: a function of two knobs that
     the models know nothing of, in place of the hardware)
  5. the gradient of the advantage-weighted log-likelihood      ml2_logprob_grad
  6. carried on to the table, candidates added in their order   ml2_embed_grad
and every call stays on the device.

With --width W the learned number is that of a small network instead: a row of W
numbers for each pair, normalised, times a vector.  Its rounds go on with
  5a. the gradients of the norm's rows, weight and bias         ml2_layer_norm_grad
  7.  the norm of all gradients, and how far to cut them        ml2_grad_norm
  8.  the parameters' step                                      ml2_adamw
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import gen  # noqa: E402
from paper_2411_10764_amd import ml2  # noqa: E402

KNOBS = 9  # values of a knob column: 0 .. 8


def measure(X, rows):
    """Stands for profiling: best at one pair of the first two knobs' values."""
    a, b = X[rows, 0], X[rows, 1]
    return -((a - 6.0).square() + (b - 2.0).square()) / 16.0


class Network:
    """One number for each of n candidates: the layer norm of the row of a table that the
    candidate's family names, times a vector.  Steps are AdamW's, on gradients cut to a norm of 1."""

    def __init__(self, n, families, width, rate, seed=1, state_bits=32):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        self.rate = rate
        self.table, self.head = normal(families, width), normal(width) * 0.1
        self.weight, self.bias = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        f32 = torch.float32
        self.lookup = ml2.Embedding(n, width, f32)
        self.norm = ml2.LayerNorm(n, width, f32)
        self.norm_grad = ml2.LayerNormGrad(n, width, f32)
        self.table_grad = ml2.EmbeddingGrad(n, families, width, f32)
        self.head_grad = torch.empty_like(self.head)
        self.dout = torch.empty(n, width, device="cuda")
        params = [self.table, self.weight, self.bias, self.head]
        grads = [self.table_grad.grad, self.norm_grad.dweight, self.norm_grad.dbias, self.head_grad]
        self.count = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.cut = ml2.GradNorm(grads, max_norm=1.0, step=self.count)
        self.adam = ml2.AdamW(params, grads, state_bits, weight_decay=[0.01, 0.0, 0.0, 0.01],
                              seed=seed)

    def forward(self, family):
        """[n] numbers; what backward needs stays in this object's buffers."""
        x = self.lookup.run(self.table, family)
        out, _, _ = self.norm.run(x, self.weight, self.bias)
        return torch.mv(out, self.head)

    def backward(self, family, dy):
        """The gradients of sum(dy * forward(family)), to their buffers."""
        norm = self.norm
        torch.mul(dy[:, None], self.head, out=self.dout)
        torch.mv(norm.out.t(), dy, out=self.head_grad)
        dx, _, _ = self.norm_grad.run(self.lookup.out, self.dout, self.weight, norm.mean,
                                      norm.rstd)
        self.table_grad.run(dx, family)

    def step(self):
        """Towards smaller values of what the gradients are of."""
        _, factor = self.cut.run()
        self.adam.run(self.rate, self.count, factor)


def run(rounds=30, draws=256, temperature=1.0, rate=4.0, seed=1, width=0):
    """Mean measurement of each round's draws."""
    w = gen.WORKLOADS["tiny"]
    X = torch.from_numpy(w.features()).to("cuda")
    v, p = ml2.ml2_load_ensemble(w.validity()), ml2.ml2_load_ensemble(w.perf())
    n = w.n
    valid = torch.empty(n, dtype=torch.uint8, device="cuda")
    margin, score = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ml2.ml2_score(v, p, X, valid, margin, score)
    score.masked_fill_(valid == 0, 0.0)  # the mask excludes them, not the score

    family = (X[:, 0] * KNOBS + X[:, 1]).to(torch.int32)
    network = Network(n, KNOBS * KNOBS, width, 0.02, seed) if width else None
    table = torch.zeros(KNOBS * KNOBS, 1, device="cuda")
    lookup = ml2.Embedding(n, 1, torch.float32)
    sampler = ml2.Sampler(1, n, draws)
    likelihood = ml2.LogProb(1, n, draws, grad_dtype=torch.float32)
    gradient = ml2.EmbeddingGrad(n, KNOBS * KNOBS, 1, torch.float32)
    T = torch.full((1,), temperature, device="cuda")
    top_p = torch.full((1,), 0.98, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    means = []
    for _ in range(rounds):
        if network:
            logits = (score + network.forward(family)).view(1, n)
        else:
            logits = (score[:, None] + lookup.run(table, family)).view(1, n)
        u = torch.rand(1, draws, generator=g, device="cuda")
        idx, _ = sampler.run(logits, u, valid, T, top_p=top_p)
        reward = measure(X, idx[0].long())
        advantage = ((reward - reward.mean()) / draws)[None].contiguous()
        _, dlogits = likelihood.run_grad(logits, idx, advantage, valid, T)
        if network:
            network.backward(family, -dlogits[0])
            network.step()
        else:
            table += rate * gradient.run(dlogits.view(n, 1), family)
        means.append(reward.mean())
    v.free()
    p.free()
    return torch.stack(means).cpu().tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rounds", type=int, default=30)
    ap.add_argument("--draws", type=int, default=256)
    ap.add_argument("--width", type=int, default=0, help="of the network's rows (0: no network)")
    a = ap.parse_args()
    for i, m in enumerate(run(a.rounds, a.draws, width=a.width)):
        print(f"round {i + 1}: mean measurement {m:.4f}")


if __name__ == "__main__":
    main()
