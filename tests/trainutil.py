"""The operators of a training step in 64 bits on the CPU, and how far float32 may be from them.

U is half a step of float32, ROUND half a step of each type relative to a value, TINY the half of
its smallest denormal.  DEPTH bounds how many additions a term of a row's sum goes through: at most
64 of a lane's own, 6 over a wave and 16 over a workgroup or over a row's pieces."""
import numpy as np
import torch

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
DEPTH = 90
BLOCK = 256


def wide(x):
    return None if x is None else x.detach().cpu().double().numpy()


# from here on a value rounds to infinity
OVER = {torch.float32: 2.0 ** 128 * (1 - 2.0 ** -25), torch.bfloat16: 2.0 ** 128 * (1 - 2.0 ** -9),
        torch.float16: 65520.0}


def close(got, want, tol, dtype):
    """Whether every value is within tol, and infinite where the type does not reach so far."""
    low, high = np.abs(want) - tol, np.abs(want) + tol
    over = np.isinf(got) & (np.sign(got) == np.sign(want)) & (high >= OVER[dtype])
    with np.errstate(invalid="ignore"):
        near = (np.abs(got - want) <= tol) & (low < OVER[dtype])
    return np.all(near | over)


# ---- layer norm ---------------------------------------------------------------

def layer_norm(x, w, b, eps):
    """(out, mean, rstd, xhat) of float64 rows"""
    mean = x.mean(1, keepdims=True)
    var = np.square(x - mean).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    xhat = (x - mean) * rstd
    y = xhat * (1.0 if w is None else w) + (0.0 if b is None else b)
    return y, mean[:, 0], rstd[:, 0], xhat


def layer_norm_tolerance(x, w, xhat, y, rstd, dtype):
    """(of out, of mean, of rstd).

    m0, the first mean, is off by at most DEPTH u avg|x|; d = x - m0 is rounded once (u |d|).
    delta = avg d is off by (DEPTH + 2) u avg|d|, avg|d| <= sigma + |delta|, and d - delta is
    rounded once more.  With sigma rstd <= 1 the centred value times rstd is off by
    2 u |xhat| + (DEPTH + 2) u, and by what the terms with |delta| <= DEPTH u avg|x| bring, all of
    second order: (DEPTH + 4) DEPTH u^2 avg|x| rstd.  The mean of squares is off by
    (DEPTH + 2) u relative, so rstd by half of that and by the roundings of the sum with eps, the
    root and the quotient: (DEPTH / 2 + 4) u.  Two more roundings make the product with the weight
    and the sum with the bias."""
    w = 1.0 if w is None else np.abs(w)
    far = (DEPTH + 4) * DEPTH * U * U * np.abs(x).mean(1)
    root = (DEPTH / 2 + 4) * U
    out = w * (np.abs(xhat) * (4 * U + root) + (DEPTH + 3) * U + (far * rstd)[:, None]) \
        + 2 * U * np.abs(y)
    sigma = np.square(x - x.mean(1, keepdims=True)).mean(1) ** 0.5
    mean = U * np.abs(x.mean(1)) + (DEPTH + 3) * U * sigma + far
    return (1 + ROUND[dtype]) * out + ROUND[dtype] * np.abs(y) + TINY[dtype], mean + 1e-44, \
        root * rstd


def layer_norm_grad(x, dout, w, rstd):
    """(dx, dweight, dbias, xhat) for the rows' own means and the given rstd"""
    xhat = (x - x.mean(1, keepdims=True)) * rstd[:, None]
    g = dout if w is None else dout * w
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True)
                          - xhat * (g * xhat).mean(1, keepdims=True))
    return dx, (dout * xhat).sum(0), dout.sum(0), xhat


def layer_norm_grad_tolerance(x, dout, w, rstd, dx, dweight, dbias, dtype, grad_dtype):
    """As above: xhat is off by 3 u |xhat| + (DEPTH + 2) u s with s = avg|x - m| rstd (the given
    rstd may be another than the row's), the averages of g and g xhat by (DEPTH + 4) u of
    the averages of their sizes and, the second, by what xhat is off times avg|g|.  A sum over
    rows goes through at most as many additions as there are rows, and 40 more for what the groups
    and workgroups leave."""
    xhat = (x - x.mean(1, keepdims=True)) * rstd[:, None]
    g = np.abs(dout if w is None else dout * w)
    s = np.abs(xhat).mean(1, keepdims=True)
    far = ((DEPTH + 4) * DEPTH * U * U * np.abs(x).mean(1) * rstd)[:, None]
    off = 3 * U * np.abs(xhat) + (DEPTH + 2) * U * s + far
    g_avg, along = g.mean(1, keepdims=True), (g * np.abs(xhat)).mean(1, keepdims=True)
    along_off = (DEPTH + 6) * U * along + (g * off).mean(1, keepdims=True)
    tol = rstd[:, None] * (4 * U * (g + g_avg + np.abs(xhat) * along) + (DEPTH + 4) * U * g_avg
                           + np.abs(xhat) * along_off + off * along)
    n = len(x) + 40
    dw = n * U * np.abs(dout * xhat).sum(0) + (np.abs(dout) * off).sum(0)
    db = n * U * np.abs(dout).sum(0)
    r, t = ROUND[grad_dtype], TINY[grad_dtype]
    return ((1 + ROUND[dtype]) * tol + ROUND[dtype] * np.abs(dx) + TINY[dtype],
            (1 + r) * dw + r * np.abs(dweight) + t, (1 + r) * db + r * np.abs(dbias) + t)


# ---- AdamW -----------------------------------------------------------------------

def adamw(p, g, m, v, lr, b1, b2, eps, decay, step, factor=1.0):
    """(p', m', v', update) in float64"""
    g = g * factor
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    up = lr / (1 - b1 ** step) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** step) + eps)
    return p - (lr * decay * p + up), m, v, up


def adamw_tolerance(p, g, m0, v0, lr, b1, b2, decay, factor, new, dtype, exact_state=True):
    """(of p', m', v').  g factor, the constants and the products are rounded once each, so m'
    is off by 5 u (b1 |m| + (1 - b1) |g|), v', a sum of sizes, by 6 u v'; the root halves that.
    The rates, the root, the product with it, the sum with eps, the product with m' and the
    quotient add 8 u relative, and decay p 3 u."""
    p1, m1, v1, up = new
    gs = np.abs(g) * abs(factor)
    m_size = b1 * np.abs(m0) + (1 - b1) * gs
    m_off = 5 * U * m_size + 2.0 ** -149
    with np.errstate(divide="ignore", invalid="ignore"):
        worse = np.where(m1 != 0, m_off / np.abs(m1), 0.0)
    up_off = np.abs(up) * (worse + 12 * U)
    tol = up_off + 3 * U * lr * abs(decay) * np.abs(p) + 2 * U * np.abs(p1) + 1e-44
    v_off = 6 * U * v1 + 2.0 ** -148
    return tol * (1 + ROUND[dtype]) + ROUND[dtype] * np.abs(p1) + TINY[dtype], m_off, v_off


# ---- states in 8 bits ---------------------------------------------------------------

PHI, PLASTIC, LOW = 0x9E3779B9, 0xC13FA9A9, 0xFFFFFFFF


def _fold(k, word):
    k = (k + word + PHI) & LOW
    k ^= k >> 16
    k = k * PHI & LOW
    k ^= k >> 15
    k = k * PLASTIC & LOW
    return k ^ (k >> 16)


def hashed(seed, step, place, index):
    """32 bits for every index (an int64 array whose upper halves are all the same)"""
    k = 0
    for word in (seed & LOW, seed >> 32, step & LOW, place):
        k = _fold(k, word)
    high = int(index[0]) >> 32 if len(index) else 0
    if high:
        k = _fold(k, high)
    h = (np.uint64(k) + (index.astype(np.uint64) & np.uint64(LOW)) * np.uint64(PHI)) & np.uint64(LOW)
    h ^= h >> np.uint64(15)
    h = h * np.uint64(PLASTIC) & np.uint64(LOW)
    return (h ^ (h >> np.uint64(16))).astype(np.int64)


def values(codes):
    """What e4m3 codes (uint8) stand for, by the format's definition"""
    c = codes.astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    size = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where(c & 128, -size, size)


def scales(x):
    """Scales of the blocks of a float64 state"""
    n = len(x)
    top = np.zeros(-(-n // BLOCK) * BLOCK)
    top[:n] = np.abs(x)
    return np.maximum(top.reshape(-1, BLOCK).max(1) / 448, 2.0 ** -100)


def rounded(size, bits, least):
    """Codes of sizes in units of their scale, up where the part cut off and the bits say so"""
    unit = np.exp2(np.maximum(np.frexp(size)[1] - 4, -9).astype(np.float64))
    z = np.floor(size / unit + (bits * 16 + 8) / 2.0 ** 20) * unit
    z = np.where(size > 0, np.clip(z, least * 2.0 ** -9, 448.0), z)
    e = np.where(z > 0, np.maximum(np.frexp(z)[1] - 1, -6), -6)
    return (z / np.exp2(e - 3.0) + (e + 6) * 8).astype(np.int64)


def split(state, n):
    """(codes, scales) of an 8-bit state's bytes"""
    raw = state.cpu().numpy()
    k = -(-n // BLOCK) * BLOCK
    return raw[:n].copy(), raw[k:].view(np.float32).astype(np.float64)


def decoded(state, n):
    codes, scale = split(state, n)
    return values(codes) * np.repeat(scale, BLOCK)[:n]


def encode_state(x):
    """A state (bytes, on the CPU) near float64 x: codes to the nearest"""
    n, scale = len(x), scales(x).astype(np.float32)
    size = np.abs(x) / np.repeat(scale.astype(np.float64), BLOCK)[:n]
    code = rounded(size, np.full(n, 32767.5), 0) + np.where(x < 0, 128, 0)
    raw = np.zeros(-(-n // BLOCK) * BLOCK, np.uint8)
    raw[:n] = code
    return torch.from_numpy(np.concatenate([raw, scale.view(np.uint8)]))


def check_state(state, n, want, bits, least, slack, ok):
    """An 8-bit state against the float64 values it was made of, which float32 has to within `slack`
    relative (where `ok`): every scale is off by that and 4 u, and every code is the one of a value
    that is off by as much and by two more roundings."""
    codes, scale = split(state, n)
    ref = scales(want)
    tau = slack + 4 * U
    assert np.all(np.abs(scale - ref) <= tau * ref)
    size = np.abs(want) / np.repeat(ref, BLOCK)[:n]
    tau = 2 * tau + 2 * U
    low = rounded(size * (1 - tau), bits, least)
    high = rounded(size * (1 + tau), bits, least)
    got = (codes & 127).astype(np.int64)
    good = (got == low) | (got == high)
    assert np.all(good[ok]), np.nonzero(~good & ok)[0][:5]
    assert np.mean(low != high) <= max(0.01, 4 / n)  # the bits decide, not the slack
    assert np.all(((codes >= 128) == (want < 0))[ok])
