"""Drawing from a row of scores, learning from what was drawn, and the tables
that it indexes: the operators as cases to time.

A case holds sizes only.  `prepare` builds what a program has in hand (scores
of candidates or of a vocabulary, masks, given random numbers, tables, token
ids, output buffers); `run` makes one pass through one operator:

  sample   per row of scores: temperature, top-k, top-p and min-p, then draws
           from given uniform numbers
  logprob  log-probabilities of given rows under the masked softmax
  learn    the same with the gradient of their weighted sum to the scores
  embed    rows of a table, scaled
  table    the gradient of that table, tokens added in their order

With `own` the calls are those of paper_2411_10764_amd.ml2, without it the
same operators in elementary torch operations.

What a draw is, so that it can be checked to the last index: with m the best
included score and R = 1 / T, all in float32,
  z = (s - m) * R (0 where s == m),  weight q = rint(exp(z) * 2**31), an integer,
entries ordered by (score descending, index ascending); top-k keeps the first
k, top-p of those the entries before which less than ceil(p * sum) of their
weight lies, min-p those with z >= log(min_p); with M the weight kept, a
uniform u draws the first index at which the running weight of the kept
entries passes floor(u * M).  Sums of whole weights are exact in any order.
"""
import math
import types

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ONE = float(2 ** 31)  # the weight of the best entry
DEV = "cuda"


def _scores(name, call, rows, n, per, dtype, *, spread, mask=0.0, shared=False, pad=0,
            T=1.0, k=0, p=1.0, minp=0.0, mixed=False):
    return {"name": name, "call": call, "rows": rows, "n": n, "per": per, "dtype": dtype,
            "spread": spread, "mask": mask, "shared": shared, "pad": pad,
            "T": T, "k": k, "p": p, "minp": minp, "mixed": mixed}


def _table(name, call, tokens, V, D, dtype, *, skew=False, pad=0, out="same"):
    return {"name": name, "call": call, "tokens": tokens, "V": V, "D": D, "dtype": dtype,
            "skew": skew, "pad": pad, "out": out}


def listed():
    return [
        # A small proposal batch of an interactive tuning loop: 32 of 4,096
        # candidates drawn where the validity model accepts.  Launches count.
        _scores("sample_1x4k_f32_d32", "sample", 1, 4096, 32, "f32", spread=0.7, mask=0.4,
                T=0.5, k=512, p=0.95),
        # A few sequences being decoded, one token each, over a large vocabulary.
        _scores("sample_4x131k_bf16", "sample", 4, 131072, 1, "bf16", spread=2.5,
                T=0.8, k=50, p=0.9),
        # A serving batch whose requests each bring their own settings, odd vocabulary.
        _scores("sample_64x50k_f16_mixed", "sample", 64, 50021, 1, "f16", spread=2.5,
                mixed=True),
        # The largest decoding batch, top-p alone, padded rows.
        _scores("sample_256x100k_bf16", "sample", 256, 100003, 1, "bf16", spread=2.0, pad=61,
                T=0.9, p=0.95, minp=0.001),
        # The benchmark's largest pool: 1,024 candidates drawn, half the pool rejected.
        _scores("sample_1x16m_f32_d1024", "sample", 1, 16777216, 1024, "f32", spread=3.2,
                mask=0.52, T=1.0, k=262144, p=0.9),
        # Log-probabilities of 512 measured candidates of a merged space.
        _scores("logprob_1x4m_f32_d512", "logprob", 1, 4194304, 512, "f32", spread=2.2,
                mask=0.5, T=0.7),
        # The gradient of a small pool's measured rows: the batch of one round.
        _scores("learn_1x262k_f32_d128", "learn", 1, 262144, 128, "f32", spread=1.4, mask=0.4,
                T=0.7),
        # Token log-likelihoods of a training batch over a vocabulary.
        _scores("learn_4096x50k_bf16", "learn", 4096, 50021, 1, "bf16", spread=2.0, pad=3),
        # Vectors of a few drawn candidates.
        _table("embed_96x128_f32", "embed", 96, 4096, 128, "f32"),
        # A training batch's tokens.
        _table("embed_32k_x1024_bf16", "embed", 32768, 131072, 1024, "bf16", skew=True),
        # The table's gradient for such a batch, kept in 32 bits.
        _table("table_32k_x1024_bf16", "table", 32768, 131072, 1024, "bf16", skew=True,
               out="f32"),
        # One learned number per pair of knob values, gathered from a whole pool.
        _table("table_4m_x1_f32", "table", 4194304, 81, 1, "f32"),
    ]


MOST = 4096 * 50021  # entries of the largest case


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    call = rng.choice(["sample", "sample", "logprob", "learn", "embed", "table"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if call in ("embed", "table"):
        D = rng.choice([_log(rng, 1, 2048), 8 * _log(rng, 1, 256)])
        V = _log(rng, 2, max(2, min(200000, (1 << 27) // D)))
        tokens = _log(rng, 1, min(1 << 22, (1 << 25) // D))
        c = _table("", call, tokens, V, D, dtype, skew=rng.random() < 0.5,
                   pad=rng.choice([0, 0, 1, 8]), out=rng.choice(["same", "f32"]))
    else:
        most = (1 << 24) if call == "sample" else (1 << 26)
        n = _log(rng, 2, 1 << 24)
        rows = _log(rng, 1, max(1, min(8192 if call == "learn" else 512, most // n)))
        per = 1 if rng.random() < 0.5 else _log(rng, 1, max(1, min(1024, n, 4096 // rows)))
        c = _scores("", call, rows, n, per, dtype,
                    spread=rng.uniform(1.0, 3.0) if n < (1 << 20) else rng.uniform(2.0, 3.5),
                    mask=rng.choice([0.0, 0.4, 0.9]), shared=rng.random() < 0.3,
                    pad=rng.choice([0, 0, 1, 13, 64]), T=rng.choice([0.3, 0.7, 1.0]),
                    k=rng.choice([0, 1, 50, 1000]), p=rng.choice([1.0, 0.95, 0.8, 0.3]),
                    minp=rng.choice([0.0, 0.0, 0.05]),
                    mixed=call == "sample" and rng.random() < 0.3)
    del c["name"]
    return c


def work(c):
    b = SIZE[c["dtype"]]
    if c["call"] in ("embed", "table"):
        moved = c["tokens"] * c["D"]
        if c["call"] == "embed":
            distinct = min(c["tokens"], c["V"])  # rows of the table read at least once
            return {"bytes": b * (distinct * c["D"] + moved) + 4 * c["tokens"], "flops": moved}
        o = 4 if c["out"] == "f32" else b
        return {"bytes": b * moved + 4 * c["tokens"] + o * c["V"] * c["D"], "flops": moved}
    entries = c["rows"] * c["n"]
    mask = 0 if not c["mask"] else c["n"] if c["shared"] else entries
    size = b * entries * (2 if c["call"] == "learn" else 1)
    # a score is compared, shifted, scaled, exponentiated (about 8) and summed
    return {"bytes": size + mask + 12 * c["rows"] * c["per"],
            "flops": entries * (16 if c["call"] == "learn" else 12)}


# ---- inputs -----------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _param(c, name, values, g, dtype):
    """A setting of every row: the case's own, or, where rows are mixed, one of `values`."""
    if not c["mixed"]:
        return torch.full((c["rows"],), c[name], dtype=dtype, device=DEV)
    at = torch.randint(len(values), (c["rows"],), generator=g, device=DEV)
    return torch.tensor(values, dtype=dtype, device=DEV)[at]


def prepare(c, seed):
    g = _generator(seed)
    s = types.SimpleNamespace(call=c["call"], dtype=DTYPES[c["dtype"]])
    if c["call"] in ("embed", "table"):
        N, V, D = c["tokens"], c["V"], c["D"]
        s.N, s.V, s.D = N, V, D
        if c["skew"]:  # frequent tokens first, as in text
            u = torch.rand(N, generator=g, device=DEV)
            s.ids = (torch.exp(u * math.log(V + 1.0)) - 1).to(torch.int32).clamp_(0, V - 1)
        else:
            s.ids = torch.randint(V, (N,), generator=g, device=DEV, dtype=torch.int32)
        s.ids[torch.rand(N, generator=g, device=DEV) < 0.01] = -1  # padding
        s.scale = math.sqrt(D)
        s.out_dtype = torch.float32 if c["call"] == "table" and c["out"] == "f32" else s.dtype
        if c["call"] == "embed":
            s.table = torch.randn(V, D + c["pad"], generator=g, device=DEV).to(s.dtype)[:, :D]
        else:
            s.dout = torch.randn(N, D + c["pad"], generator=g, device=DEV).to(s.dtype)[:, :D]
        if own:
            from paper_2411_10764_amd import ml2
            s.plan = (ml2.Embedding(N, D, s.dtype) if c["call"] == "embed" else
                      ml2.EmbeddingGrad(N, V, D, s.out_dtype))
        return s
    rows, n, d = c["rows"], c["n"], c["per"]
    s.rows, s.n, s.d = rows, n, d
    x = torch.randn(rows, n + c["pad"], generator=g, device=DEV).mul_(c["spread"])
    s.scores = x.to(s.dtype)[:, :n]
    del x
    s.valid = None
    if c["mask"]:
        shape = (n,) if c["shared"] else (rows, n)
        s.valid = (torch.rand(shape, generator=g, device=DEV) >= c["mask"]).to(torch.uint8)
        s.valid[..., 0] = 1
    s.T = _param(c, "T", [0.0, 0.3, 0.7, 1.0, 1.2], g, torch.float32)
    if c["call"] == "sample":
        s.k = _param(c, "k", [0, 1, 20, 50, 1000], g, torch.int32)
        s.p = _param(c, "p", [1.0, 0.95, 0.9, 0.5], g, torch.float32)
        s.minp = _param(c, "minp", [0.0, 0.02, 0.1], g, torch.float32)
        s.u = torch.rand(rows, d, generator=g, device=DEV)
    else:
        s.targets = torch.randint(n, (rows, d), generator=g, device=DEV, dtype=torch.int32)
        if d > 4:
            s.targets[:, 1] = s.targets[:, 0]  # a row measured twice
            s.targets[:, 2] = -1               # padding of a short selection
        if s.valid is not None:  # measured rows were accepted ones: else the first
            ok = s.valid.expand(rows, n).gather(1, s.targets.clamp(min=0).long())
            s.targets = torch.where(ok != 0, s.targets, torch.where(s.targets < 0, -1, 0))
            s.targets = s.targets.to(torch.int32)
        s.weight = torch.randn(rows, d, generator=g, device=DEV)
    if own:
        from paper_2411_10764_amd import ml2
        s.plan = (ml2.Sampler(rows, n, d) if c["call"] == "sample" else
                  ml2.LogProb(rows, n, d, grad_dtype=s.dtype if c["call"] == "learn" else None))
    return s


# ---- one pass ---------------------------------------------------------------

def run(s):
    if not own:
        return _PLAIN[s.call](s)
    if s.call == "sample":
        return s.plan.run(s.scores, s.u, s.valid, s.T, s.k, s.p, s.minp)
    if s.call == "logprob":
        return s.plan.run(s.scores, s.targets, s.valid, s.T)
    if s.call == "learn":
        return s.plan.run_grad(s.scores, s.targets, s.weight, s.valid, s.T)
    if s.call == "embed":
        return s.plan.run(s.table, s.ids, s.scale)
    return s.plan.run(s.dout, s.ids, s.scale)


def _included(s):
    """(scores in 32 bits with -inf where not included, the best of each row)"""
    x = s.scores.float() + 0.0
    out = torch.isnan(x)
    if s.valid is not None:
        out = out | (s.valid == 0)
    x = x.masked_fill(out, -math.inf)
    return x, x.amax(1, keepdim=True)


def _shifted(x, m, R):
    z = torch.where(x == m, torch.zeros_like(x), (x - m) * R)
    return z.masked_fill(x == -math.inf, -math.inf)


def _plain_sample(s):
    x, m = _included(s)
    greedy = ~(s.T > 0)
    R = torch.where(greedy, torch.ones_like(s.T), 1.0 / s.T)[:, None]
    z = _shifted(x, m, R)
    q = (torch.exp(z) * ONE).round().long()
    k = torch.where(greedy, torch.ones_like(s.k), s.k)
    k = torch.where(k <= 0, torch.full_like(k, s.n), k)[:, None]
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    first = torch.arange(s.n, device=DEV)[None] < k
    ordered = q.gather(1, order) * first
    upto = ordered.cumsum(1)
    share = torch.ceil(s.p.double()[:, None] * upto[:, -1:].double())
    share = torch.where(s.p[:, None] < 1.0, share.clamp(min=1.0), math.inf)
    first &= (upto - ordered) < share
    kept = torch.zeros_like(first).scatter_(1, order, first)
    kept &= z >= torch.where(s.minp > 0, s.minp.clamp(max=1.0).log(), -math.inf)[:, None]
    upto = (q * kept).cumsum(1)
    M = upto[:, -1:]
    at = torch.minimum(torch.floor(s.u.double() * M.double()).long(), M - 1)
    idx = torch.searchsorted(upto, at, right=True)
    none = (M <= 0).expand_as(idx)
    logp = z.gather(1, idx.clamp(max=s.n - 1)) - torch.log(M.float() / ONE)
    return idx.int().masked_fill(none, -1), logp.masked_fill(none, -math.inf)


def _plain_logprob(s, grad=False):
    x, m = _included(s)
    R = torch.where(s.T > 0, 1.0 / s.T, torch.ones_like(s.T))[:, None]
    z = _shifted(x, m, R)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    inside = (s.targets >= 0) & (s.targets < s.n)
    at = torch.where(inside, s.targets, 0).long()
    zt = z.gather(1, at)
    logp = torch.where(inside, torch.where(zt == -math.inf, zt, zt - torch.log(total)), 0.0)
    if not grad:
        return logp
    w = torch.where(inside & (zt != -math.inf), s.weight, 0.0)
    d = e.mul_(w.sum(1, keepdim=True) / -total)
    d = d.scatter_add_(1, at, w).mul_(R)
    return logp, d.to(s.dtype)


def _plain_embed(s):
    inside = (s.ids >= 0) & (s.ids < s.V)
    rows = s.table[torch.where(inside, s.ids, 0).long()].float() * s.scale
    return rows.masked_fill(~inside[:, None], 0.0).to(s.dtype)


def _plain_table(s):
    inside = (s.ids >= 0) & (s.ids < s.V)
    # A token of many positions is added up in several parts (32 bits hold a
    # sum of many thousand terms less exactly than one of their sums).
    parts = max(1, min(256, s.N // s.V, (1 << 22) // (s.V * s.D)))
    at = torch.arange(s.N, device=DEV) % parts * (s.V + 1)
    at = at + torch.where(inside, s.ids, s.V)
    t = torch.zeros(parts * (s.V + 1), s.D, device=DEV).index_add_(0, at, s.dout.float())
    t = t.view(parts, s.V + 1, s.D).sum(0) if parts > 1 else t
    return (t[: s.V] * s.scale).to(s.out_dtype)


_PLAIN = {"sample": _plain_sample, "logprob": _plain_logprob,
          "learn": lambda s: _plain_logprob(s, True), "embed": _plain_embed,
          "table": _plain_table}


# ---- the definition in 64 bits ----------------------------------------------

def exact(c, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = kept
    if c["call"] == "embed":
        t = torch.cat([s.table.double() * s.scale,
                       torch.zeros(1, s.D, dtype=torch.float64, device=DEV)])
        ids = s.ids.long()
        return t[torch.where((ids < 0) | (ids >= s.V), s.V, ids)]
    if c["call"] == "table":
        t = torch.zeros(s.V, s.D, dtype=torch.float64, device=DEV)
        ok = torch.nonzero((s.ids >= 0) & (s.ids < s.V))[:, 0]
        for part in ok.split(max(1, (1 << 26) // s.D)):
            t.index_put_((s.ids[part].long(),), s.dout[part].double(), accumulate=True)
        return t * s.scale
    each = [_exact_row(s, r) for r in range(s.rows)]
    return torch.stack(each) if c["call"] == "logprob" else tuple(
        torch.stack(v) for v in zip(*each))


def _exact_row(s, r):
    """One row: the included entries alone, in 64 bits."""
    x = s.scores[r]
    ok = ~torch.isnan(x) & (x != -math.inf)
    if s.valid is not None:
        ok &= (s.valid if s.valid.dim() == 1 else s.valid[r]) != 0
    at = torch.nonzero(ok)[:, 0]
    T = float(s.T[r])
    if s.call == "sample":
        return _exact_draws(s, r, x[at].float(), at, T)
    v = x[at].double() / (T if T > 0 else 1.0)
    lse = torch.logsumexp(v, 0)
    t = s.targets[r].long()
    inside = (t >= 0) & (t < s.n)
    z = torch.full((s.n,), -math.inf, dtype=torch.float64, device=DEV)
    z[at] = v - lse
    logp = torch.where(inside, z[t.clamp(0, s.n - 1)], 0.0)
    if s.call == "logprob":
        return logp
    w = torch.where(inside & (logp != -math.inf), s.weight[r].double(), 0.0)
    d = -w.sum() * torch.exp(z)
    d.index_put_((t.clamp(0, s.n - 1),), w, accumulate=True)
    return logp, d / (T if T > 0 else 1.0)


def _exact_draws(s, r, x, at, T):
    k, p, minp = int(s.k[r]), float(s.p[r]), float(s.minp[r])
    if not T > 0:
        T, k = 1.0, 1
    if not len(at):
        return (torch.full((s.d,), -1, dtype=torch.int32, device=DEV),
                torch.full((s.d,), -math.inf, dtype=torch.float64, device=DEV))
    # the definition's float32 exponents; everything after them in 64 bits
    z = (x - x.max()) * (1.0 / torch.tensor(T, dtype=torch.float32, device=DEV))
    z = z.double()
    q = torch.exp(z).mul(ONE).round()
    # (score, index) order: entries come in index order, so stable by -score
    by = torch.argsort(-x.double(), stable=True)
    if 0 < k < len(by):
        by = by[:k]
    if p < 1.0:
        before = torch.cat([q.new_zeros(1), q[by].cumsum(0)])
        need = max(1.0, math.ceil(p * float(before[-1])))
        by = by[: int((before[:-1] < need).sum())]
    by = by.sort().values
    if minp > 0:
        by = by[z[by] >= math.log(min(minp, 1.0))]
    upto = q[by].cumsum(0)
    M = float(upto[-1])
    pick = by[torch.searchsorted(upto, torch.floor(s.u[r].double() * M).clamp(max=M - 1),
                                 right=True)]
    return at[pick].int(), z[pick] - math.log(M / ONE)
