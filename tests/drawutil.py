"""Plain 64-bit forms of the operators over rows of scores and over tables, on
the CPU: one row, one entry, one token after the other."""
import math

import numpy as np

ONE = 2.0 ** 31


def as_float(x):
    """float32 numpy values of a torch tensor of any of the operators' types."""
    return x.detach().cpu().float().numpy()


def included(x, valid):
    ok = ~np.isnan(x) & (x != -np.inf)
    return ok if valid is None else ok & (np.asarray(valid) != 0)


def exponents(x, ok, T):
    """z of the included entries as defined (float32 operations); -inf elsewhere."""
    z = np.full(x.shape, -np.inf, np.float32)
    if not ok.any():
        return z
    with np.errstate(all="ignore"):
        m = x[ok].max()
        r = np.float32(1.0) / np.float32(T) if T > 0 else np.float32(1.0)
        d = (x - m).astype(np.float32) * r
    z[ok] = np.where(x[ok] == m, np.float32(0.0), d[ok])
    return z


def sample_row(x, valid, T, k, p, minp, u, lean=0.0):
    """(idx, logprob, sure) of one row's draws by the definition, exp taken in
    64 bits.  `lean` moves top-p's share by that part of the
    weight that is not exact (all but the best score's).  A draw
    is sure where its neighbours lie further off than what the float32 exp
    (1 ulp) and the rounding of a weight (1) may move."""
    x = np.asarray(x, np.float32)
    ok = included(x, valid)
    d = len(u)
    if not ok.any():
        return np.full(d, -1), np.full(d, -np.inf), np.ones(d, bool)
    if not T > 0:
        k = 1
    z = exponents(x, ok, T).astype(np.float64)
    with np.errstate(all="ignore"):
        q = np.where(ok & ~np.isnan(z), np.rint(np.exp(z) * ONE), 0.0)
    q = np.nan_to_num(q)
    at = np.nonzero(ok)[0]
    order = at[np.argsort(-x[at].astype(np.float64), kind="stable")]
    if k > 0:
        order = order[:k]
    if p < 1.0:
        before = np.concatenate([[0.0], np.cumsum(q[order])])
        share = max(1.0, math.ceil(max(0.0, float(p)) * before[-1])
                    + lean * q[order][z[order] < 0].sum())
        order = order[before[:-1] < share]
    if minp > 0:
        order = order[z[order] >= min(0.0, math.log(min(float(minp), 1.0)) - 1e-6 * lean)]
    kept = np.sort(order)
    upto = np.cumsum(q[kept])
    M = upto[-1]
    want = np.minimum(np.floor(np.asarray(u, np.float64) * M), M - 1)
    pick = np.searchsorted(upto, want, side="right")
    low = np.where(pick > 0, upto[pick - 1], 0.0)
    high = upto[pick]
    # weights other than the best score's may be off by 1 ulp and 1: a border
    # moves by those before it, floor(u * M) by u times those of the row
    off = np.cumsum(np.where(z[kept] < 0, q[kept] * 2.0 ** -23 + 1, 0.0))
    moves = off[pick] + np.asarray(u, np.float64) * off[-1]
    sure = ((low == 0) | (want - low >= moves)) & ((high == M) | (high - want > moves))
    return kept[pick], z[kept[pick]] - math.log(M / ONE), sure


def sample(x, valid, T, k, p, minp, u):
    """Rows of sample_row; a draw is sure if it is the same at either lean of
    top-p's share."""
    idx, logp, sure = [], [], []
    for r in range(x.shape[0]):
        v = None if valid is None else valid if valid.ndim == 1 else valid[r]
        a = sample_row(x[r], v, T[r], k[r], p[r], minp[r], u[r])
        lean = [sample_row(x[r], v, T[r], k[r], p[r], minp[r], u[r], s * 2.0 ** -22)
                for s in (-1, 1)]
        idx.append(a[0])
        logp.append(a[1])
        sure.append(a[2] & (lean[0][0] == a[0]) & (lean[1][0] == a[0]))
    return np.stack(idx), np.stack(logp), np.stack(sure)


def logprob_row(x, valid, T, targets, weight=None):
    """(logprob, gradient) of one row in 64 bits; a log-probability beyond
    float32's range is -inf, as a float32 holds it."""
    n = len(x)
    ok = included(x, valid)
    T = float(T) if T > 0 else 1.0
    z = np.full(n, -np.inf)
    if ok.any():
        v = x[ok].astype(np.float64)
        m = v.max()
        with np.errstate(all="ignore"):
            z[ok] = np.where(v == m, 0.0, (v - m) / T)
        z -= math.log(np.exp(z).sum())
    logp = np.zeros(len(targets))
    grad = np.zeros(n)
    total = 0.0
    for j, t in enumerate(targets):
        if not 0 <= t < n:
            continue
        logp[j] = z[t]
        if weight is not None and ok[t]:
            grad[t] += float(weight[j])
            total += float(weight[j])
    grad -= total * np.exp(z)
    logp[logp < -np.finfo(np.float32).max] = -np.inf
    return logp, grad / T


def gradient_tolerance(x, valid, T, targets, weight, round_to, tiny):
    """What a float32 computation of one row's gradient may be off by.

    The two terms of an entry are p * W / T and the weights of the targets that
    name it / T.  An exponent z is two float32 roundings from its value and the
    exponential adds one, (|z| + 2) 2^-23 of p, and the sum that p is divided by
    is within 330 * 2^-23 of its value: 8e-5 of both terms, which also covers
    the sums of weights.  A p below 2^-125 may be taken as 0.  `round_to` and
    `tiny`: half an ulp of the result's type, relative, and where that ends."""
    ok = included(x, valid)
    t = float(T) if T > 0 else 1.0
    w = np.where([0 <= j < len(x) and bool(ok[j]) for j in targets],
                 np.abs(np.asarray(weight, np.float64)), 0.0)
    z = np.full(len(x), -np.inf)
    if ok.any():
        v = x[ok].astype(np.float64)
        with np.errstate(all="ignore"):
            z[ok] = np.where(v == v.max(), 0.0, (v - v.max()) / t)
        z -= math.log(np.exp(z).sum())
    with np.errstate(over="ignore"):
        size = np.exp(z) * w.sum() / t
        for j, q in zip(targets, w):
            if 0 <= j < len(x):
                size[j] += q / t
        _, want = logprob_row(x, valid, T, targets, weight)
        return 8e-5 * size + 2.0 ** -125 * w.sum() / t + round_to * np.abs(want) + tiny


def check_gradient(got, x, valid, T, targets, weight, round_to, tiny, most):
    """Asserts that `got` is the gradient of logprob_row, row by row: within the
    tolerance at every entry (a NaN is within none), infinite only where the
    value passes `most`, the largest number of its type, and 0 at an entry that
    is not included."""
    for r in range(x.shape[0]):
        v = None if valid is None else valid if valid.ndim == 1 else valid[r]
        with np.errstate(over="ignore"):
            _, want = logprob_row(x[r], v, T[r], targets[r], weight[r])
        assert not np.isnan(want).any(), "the formula itself has no value here"
        ok = included(x[r], v)
        assert np.all(got[r][~ok] == 0.0), (r, "not included", np.nonzero(got[r][~ok] != 0)[0][:5])
        tol = gradient_tolerance(x[r], v, T[r], targets[r], weight[r], round_to, tiny)
        with np.errstate(invalid="ignore"):
            near = np.abs(got[r].astype(np.float64) - want) <= tol
        beyond = np.isinf(got[r]) & (np.sign(got[r]) == np.sign(want)) & (np.abs(want) + tol > most)
        bad = ~(near & np.isfinite(got[r]) | beyond)
        assert not bad.any(), (r, np.nonzero(bad)[0][:5], got[r][bad][:5], want[bad][:5])


def embed(table, ids, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for i, v in enumerate(ids):
        if 0 <= v < table.shape[0]:
            out[i] = table[v].astype(np.float64) * scale
    return out


def embed_grad(dout, ids, V, scale):
    out = np.zeros((V, dout.shape[1]))
    ok = (ids >= 0) & (ids < V)
    np.add.at(out, ids[ok], dout[ok].astype(np.float64))
    return out * scale
