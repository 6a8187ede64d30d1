"""What a training step holds besides its products, its loss and its tables:
layer norm with its gradient, the norm that gradients are cut to, and the
optimizer's step, as cases to time.

A case holds sizes only.  `prepare` builds what a program has in hand
(activations, gradients, parameters, states, output buffers); `run` makes one
pass through one operator:

  ln       rows normalised, scaled and shifted, with their statistics
  ln_grad  the gradients of the rows, the weight and the bias
  clip     the norm of many gradients together, and what to multiply them by
  adamw    a step of AdamW over many tensors, states in 32 or in 8 bits

With `own` the calls are those of paper_2411_10764_amd.ml2, without it the
same operators in elementary torch operations.

What a step is, so that it can be checked (float32 throughout):
  g = grad * grad_scale,  m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g g
  p' = p - (lr decay p + lr / (1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps))
States in 8 bits are m and r = sqrt(v) as e4m3 numbers, each block of 256
elements of a tensor with a scale of its own, max(largest / 448, 2^-100).  They
are rounded up or down at random, so that slow averages move at all: with k the
20 bits below the last one kept and h(seed, step, tensor, element) 32 hashed
bits, up where k + 16 * (16 bits of h) + 8 passes 2^20.  An r that is not 0
never becomes 0.
"""
import itertools
import math
import types

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda"
EPS = 1e-5
LR, B1, B2, ADAM_EPS, DECAY, STEP, SEED = 1e-3, 0.9, 0.999, 1e-8, 0.1, 1000, 5
BLOCK = 256  # elements that share a scale


def _norm(name, call, rows, width, dtype, params, *, pad=0, bias=True):
    return {"name": name, "call": call, "rows": rows, "width": width, "dtype": dtype,
            "params": params, "pad": pad, "bias": bias}


def _tensors(name, call, count, total, grad, *, param="f32", bits=32, copy=False, gap=0,
             scaled=False, decay="all"):
    return {"name": name, "call": call, "count": count, "total": total, "grad": grad,
            "param": param, "bits": bits, "copy": copy, "gap": gap, "scaled": scaled,
            "decay": decay}


def listed():
    return [
        # The vectors of a few drawn candidates.  Launches count.
        _norm("ln_96x128_f32", "ln", 96, 128, "f32", "f32"),
        # A training batch's tokens, parameters kept in 32 bits.
        _norm("ln_32k_x1024_bf16", "ln", 32768, 1024, "bf16", "f32"),
        # Rows of scores as wide as an odd vocabulary, padded.
        _norm("ln_515x50021_f16", "ln", 515, 50021, "f16", "f16", pad=3),
        # Their gradients: the drawn candidates',
        _norm("ln_grad_96x128_f32", "ln_grad", 96, 128, "f32", "f32"),
        # the training batch's,
        _norm("ln_grad_32k_x1024_bf16", "ln_grad", 32768, 1024, "bf16", "f32"),
        # an odd width whose rows are aligned to their elements only,
        _norm("ln_grad_3001x771_f16", "ln_grad", 3001, 771, "f16", "f16", pad=6),
        # and rows too wide for one workgroup's registers.
        _norm("ln_grad_260x50021_f32", "ln_grad", 260, 50021, "f32", "f32", bias=False),
        # The gradients of a small policy: a table of pairs of knob values, some layers.
        _tensors("clip_5t_50k_f32", "clip", 5, 50000, "f32"),
        # A table of 131,072 x 1,024, its gradient in 16 bits.
        _tensors("clip_1t_134m_bf16", "clip", 1, 1 << 27, "bf16"),
        # The small policy's step.
        _tensors("adamw_5t_50k_f32", "adamw", 5, 50000, "f32", scaled=True),
        # Many tensors of all sizes in flat buffers: master parameters in 32 bits, a copy in
        # 16 bits for the next forward pass, no decay for every other tensor.
        _tensors("adamw_60t_12m_bf16_copy", "adamw", 60, 12000000, "bf16", copy=True, gap=3,
                 scaled=True, decay="some"),
        # The large table with states in 8 bits.
        _tensors("adamw_1t_134m_bf16_8bit", "adamw", 1, 1 << 27, "bf16", param="bf16", bits=8),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    call = rng.choice(["ln", "ln", "ln_grad", "ln_grad", "clip", "adamw", "adamw"])
    if call in ("ln", "ln_grad"):
        # (the rows of narrower gradients are little more than what rounding leaves)
        width = rng.choice([_log(rng, 5, 65536), 8 * _log(rng, 1, 8192)])
        rows = _log(rng, 1, max(1, min(200000, (1 << 25) // width)))
        dtype = rng.choice(["f32", "bf16", "f16"])
        c = _norm("", call, rows, width, dtype, rng.choice([dtype, "f32"]),
                  pad=rng.choice([0, 0, 1, 8]), bias=rng.random() < 0.7)
    else:
        bits = rng.choice([32, 32, 8]) if call == "adamw" else 32
        total = _log(rng, 1000, 1 << (25 if bits == 32 else 26))
        count = _log(rng, 1, 8 if bits == 8 else 150)
        param = rng.choice(["f32", "f32", "bf16", "f16"])
        c = _tensors("", call, count, total, rng.choice(["f32", "bf16", "f16"]), param=param,
                     bits=bits, copy=call == "adamw" and param == "f32" and rng.random() < 0.5,
                     gap=rng.choice([0, 1, 8]), scaled=rng.random() < 0.5,
                     decay=rng.choice(["all", "some"]))
    del c["name"]
    return c


def _sizes(c):
    """Sizes of `count` tensors that differ by up to a factor of 400, odd ones among them."""
    parts = [400.0 ** ((i * 7 % c["count"]) / c["count"]) for i in range(c["count"])]
    return [max(1, int(c["total"] * p / sum(parts))) for p in parts]


def work(c):
    if c["call"] in ("ln", "ln_grad"):
        e, b, p = c["rows"] * c["width"], SIZE[c["dtype"]], SIZE[c["params"]]
        if c["call"] == "ln":
            return {"bytes": 2 * b * e + (1 + c["bias"]) * p * c["width"] + 8 * c["rows"],
                    "flops": 8 * e}
        return {"bytes": 3 * b * e + (2 + c["bias"]) * p * c["width"] + 8 * c["rows"],
                "flops": 16 * e}
    e = sum(_sizes(c))
    if c["call"] == "clip":
        return {"bytes": SIZE[c["grad"]] * e, "flops": 2 * e}
    state = 8 if c["bits"] == 32 else 2 * (1 + 4 / BLOCK)
    moved = 2 * SIZE[c["param"]] + SIZE[c["grad"]] * (1 + c["copy"]) + 2 * state
    return {"bytes": moved * e, "flops": (20 if c["bits"] == 32 else 40) * e}


# ---- inputs -----------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _slices(flat, sizes, gap):
    """The tensors of a flat buffer, `gap` elements between each and the next."""
    ends = itertools.accumulate(n + gap for n in sizes)
    return [flat[a - gap - n: a - gap] for a, n in zip(ends, sizes)]


def prepare(c, seed):
    g = _generator(seed)
    s = types.SimpleNamespace(call=c["call"])
    if c["call"] in ("ln", "ln_grad"):
        return _prepare_norm(c, s, g)
    s.sizes = _sizes(c)
    n, s.gap = sum(s.sizes) + c["gap"] * (c["count"] - 1), c["gap"]
    on = torch.zeros(n, device=DEV)  # 0 between the tensors
    torch._foreach_add_(_slices(on, s.sizes, s.gap), 1.0)
    grad = torch.randn(n, generator=g, device=DEV).mul_(torch.rand(n, generator=g, device=DEV))
    s.grad = grad.mul_(0.01).mul_(on).to(DTYPES[c["grad"]])
    s.grads = _slices(s.grad, s.sizes, s.gap)
    if c["call"] == "clip":
        s.max_norm, s.scale = 1.0, 0.5
        if own:
            from paper_2411_10764_amd import ml2
            s.plan = ml2.GradNorm(s.grads, s.max_norm, s.scale)
        return s
    s.bits, s.scaled = c["bits"], None
    if c["scaled"]:
        s.scaled = torch.rand(1, generator=g, device=DEV).mul_(0.5).add_(0.5)
    s.decay = [DECAY if c["decay"] == "all" or i % 2 else 0.0 for i in range(c["count"])]
    s.decay_at = None
    if c["decay"] != "all":
        s.decay_at = torch.zeros(n, device=DEV)
        torch._foreach_add_(_slices(s.decay_at, s.sizes, s.gap), s.decay)
    s.param = torch.randn(n, generator=g, device=DEV).mul_(0.02).mul_(on).to(DTYPES[c["param"]])
    m = torch.randn(n, generator=g, device=DEV).mul_(0.003).mul_(on)
    r = torch.rand(n, generator=g, device=DEV).mul_(0.01).mul_(on)
    s.param_out = torch.zeros_like(s.param)
    s.copy = torch.zeros(n, dtype=s.grad.dtype, device=DEV) if c["copy"] else None
    s.copies = _slices(s.copy, s.sizes, s.gap) if c["copy"] else None
    if c["bits"] == 32:
        s.m, s.v = m, r.square_()
        s.m_out, s.v_out = torch.zeros_like(s.m), torch.zeros_like(s.v)
        states = [_slices(x, s.sizes, s.gap) for x in (s.m, s.v, s.m_out, s.v_out)]
    else:
        s.m = [_eight(x) for x in _slices(m, s.sizes, s.gap)]
        s.v = [_eight(x) for x in _slices(r, s.sizes, s.gap)]
        s.m_out, s.v_out = [torch.zeros_like(x) for x in s.m], [torch.zeros_like(x) for x in s.v]
        states = s.m, s.v, s.m_out, s.v_out
    if own:
        from paper_2411_10764_amd import ml2
        s.plan = ml2.AdamW(
            _slices(s.param, s.sizes, s.gap), s.grads, state_bits=s.bits, m=states[0],
            v=states[1], weight_decay=s.decay, betas=(B1, B2), eps=ADAM_EPS, seed=SEED,
            copies=s.copies, out=(_slices(s.param_out, s.sizes, s.gap), states[2], states[3]))
    return s


def _eight(x):
    """The 8-bit state that stands for x: its codes, then its blocks' scales."""
    n, blocks = x.numel(), -(-x.numel() // BLOCK)
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - n)).view(blocks, BLOCK)
    scale = (x.abs().amax(1) / 448).clamp(min=2.0 ** -100)
    code = (x / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.cat([code.view(-1), scale.view(torch.uint8)])


def _prepare_norm(c, s, g):
    rows, D, dtype = c["rows"], c["width"], DTYPES[c["dtype"]]
    s.rows, s.D, s.dtype = rows, D, dtype
    x = torch.randn(rows, D + c["pad"], generator=g, device=DEV)
    x.mul_(torch.rand(rows, 1, generator=g, device=DEV).mul_(3).add_(0.1))
    x.add_(torch.randn(rows, 1, generator=g, device=DEV))
    x[:, 0] *= 8  # a channel that stands out
    s.x = x.to(dtype)[:, :D]
    del x
    s.weight = (torch.randn(D, generator=g, device=DEV) * 0.2 + 1).to(DTYPES[c["params"]])
    s.bias = None
    if c["bias"]:
        s.bias = (torch.randn(D, generator=g, device=DEV) * 0.2).to(DTYPES[c["params"]])
    if c["call"] == "ln_grad":
        s.dout = torch.randn(rows, D + c["pad"], generator=g, device=DEV).to(dtype)[:, :D]
        mean, rstd = _statistics(s.x.double())
        s.mean, s.rstd = mean[:, 0].float(), rstd[:, 0].float()
    if own:
        from paper_2411_10764_amd import ml2
        s.plan = (ml2.LayerNorm(rows, D, dtype) if c["call"] == "ln" else
                  ml2.LayerNormGrad(rows, D, dtype, s.weight.dtype, bias=c["bias"]))
    return s


# ---- one pass ---------------------------------------------------------------

def run(s):
    if not own:
        return _PLAIN[s.call](s)
    if s.call == "ln":
        return s.plan.run(s.x, s.weight, s.bias, EPS)
    if s.call == "ln_grad":
        return s.plan.run(s.x, s.dout, s.weight, s.mean, s.rstd)
    if s.call == "clip":
        return s.plan.run()
    s.plan.run(LR, STEP, s.scaled)
    return _updated(s)


def _updated(s):
    if s.bits == 32:
        return s.param_out, s.copy, s.m_out, s.v_out
    return (_slices(s.param_out, s.sizes, s.gap), s.copies,
            [_views(x, n) for x, n in zip(s.m_out, s.sizes)],
            [_views(x, n) for x, n in zip(s.v_out, s.sizes)])


def _views(state, n):
    """An 8-bit state's numbers, in units of their block's scale, and the scales."""
    blocks = -(-n // BLOCK)
    return (state[:n].view(torch.float8_e4m3fn),
            state[blocks * BLOCK:].view(torch.float32))


def _statistics(x):
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    return mean, torch.rsqrt(var + EPS)


def _plain_ln(s):
    x = s.x.float()
    mean, rstd = _statistics(x)
    y = (x - mean) * rstd * s.weight.float()
    if s.bias is not None:
        y = y + s.bias.float()
    return y.to(s.dtype), mean[:, 0], rstd[:, 0]


def _plain_ln_grad(s):
    d, rstd = s.dout.float(), s.rstd[:, None]
    xhat = (s.x.float() - s.mean[:, None]) * rstd
    g = d * s.weight.float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    dweight = (d * xhat).sum(0).to(s.weight.dtype)
    return dx.to(s.dtype), dweight, None if s.bias is None else d.sum(0).to(s.weight.dtype)


def _plain_clip(s):
    norm = s.grad.float().square().sum(dtype=torch.float64).sqrt() * s.scale
    factor = torch.where(torch.isfinite(norm), s.scale * (s.max_norm / norm).clamp(max=1.0),
                         torch.nan)
    return norm.float().view(1), factor.float().view(1)


def _rates():
    """lr / (1 - b1^t) and 1 / sqrt(1 - b2^t)"""
    return LR / (1 - B1 ** STEP), 1 / math.sqrt(1 - B2 ** STEP)


def _step(s, p, grad, m, v, decay):
    """(p', m', v') of float32 values"""
    a, b = _rates()
    g = grad.float()
    if s.scaled is not None:
        g = g * s.scaled
    m = m * B1 + g * (1 - B1)
    v = v * B2 + g * (1 - B2) * g
    p = p.float()
    return p - (p * decay * LR + m * a / (v.sqrt() * b + ADAM_EPS)), m, v


def _plain_adamw(s):
    if s.bits == 32:
        decay = DECAY if s.decay_at is None else s.decay_at
        p, m, v = _step(s, s.param, s.grad, s.m, s.v, decay)
        return p.to(s.param.dtype), None if s.copy is None else p.to(s.copy.dtype), m, v
    each = zip(_slices(s.param, s.sizes, s.gap), s.grads, s.m, s.v, s.decay)
    new = [_step(s, p, g, _decoded(m, g.numel()), _decoded(v, g.numel()).square(), decay)
           for p, g, m, v, decay in each]
    hashed = [_hashed(i, n) for i, n in enumerate(s.sizes)]
    return ([x[0].to(s.param.dtype) for x in new],
            None if s.copy is None else [x[0].to(s.copy.dtype) for x in new],
            [_views(_encoded(x[1], h >> 16, 0), len(h)) for x, h in zip(new, hashed)],
            [_views(_encoded(x[2].sqrt(), h & 0xFFFF, 1), len(h)) for x, h in zip(new, hashed)])


def _decoded(state, n):
    code, scale = _views(state, n)
    return code.float() * scale.repeat_interleave(BLOCK)[:n]


def _encoded(x, bits, least):
    n, blocks = x.numel(), -(-x.numel() // BLOCK)
    rows = torch.nn.functional.pad(x, (0, blocks * BLOCK - n)).view(blocks, BLOCK)
    scale = (rows.abs().amax(1) * (1.0 / 448)).clamp(min=2.0 ** -100)
    size = (rows.abs() * (1.0 / scale)[:, None]).view(-1)[:n]
    # an e4m3 number is a float32 number 2^120 times as small without its last 20 bits
    code = ((size * 2.0 ** -120).view(torch.int32) + (bits * 16 + 8).int()) >> 20
    code = code.clamp(max=0x7E)
    if least:
        code = torch.where(x > 0, code.clamp(min=least), code)
    code = torch.where(x < 0, code + 128, code).to(torch.uint8)
    return torch.cat([torch.nn.functional.pad(code, (0, blocks * BLOCK - n)),
                      scale.view(torch.uint8)])


PHI, PLASTIC = 0x9E3779B9, 0xC13FA9A9  # 2^32 over the golden and over the plastic number
LOW = 0xFFFFFFFF


def _key(tensor):
    key = 0
    for word in (SEED & LOW, SEED >> 32, STEP, tensor):
        key = (key + word + PHI) & LOW
        key ^= key >> 16
        key = key * PHI & LOW
        key ^= key >> 15
        key = key * PLASTIC & LOW
        key ^= key >> 16
    return key


def _hashed(tensor, n):
    """32 bits for every element of a tensor (of fewer than 2^32 elements)"""
    h = (torch.arange(n, device=DEV) * PHI + _key(tensor)) & LOW
    h = h ^ (h >> 15)
    h = (h * PLASTIC) & LOW
    return h ^ (h >> 16)


_PLAIN = {"ln": _plain_ln, "ln_grad": _plain_ln_grad, "clip": _plain_clip, "adamw": _plain_adamw}


# ---- the definition in 64 bits ----------------------------------------------

def exact(c, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = kept
    if c["call"] == "clip":
        norm = s.scale * torch.linalg.vector_norm(s.grad.double())
        return norm.view(1), s.scale * (s.max_norm / norm).clamp(max=1.0).view(1)
    if c["call"] == "adamw":
        return _exact_adamw(s)
    x, w = s.x.double(), s.weight.double()
    centred = x - x.sum(1, keepdim=True) / s.D
    rstd = 1 / (centred.pow(2).sum(1, keepdim=True) / s.D + EPS).sqrt()
    if c["call"] == "ln":
        y = centred * (rstd * w)
        return y if s.bias is None else y + s.bias.double(), x.sum(1) / s.D, rstd[:, 0]
    xhat, d = centred * rstd, s.dout.double()
    # the derivative of xhat to x, applied to g = dout * weight
    g = d * w
    along = torch.linalg.vecdot(g, xhat)[:, None] / s.D
    dx = (g - (g.sum(1, keepdim=True) / s.D + xhat * along)) * rstd
    return dx, torch.einsum("rd,rd->d", d, xhat), None if s.bias is None else d.sum(0)


def _exact_adamw(s):
    parts = zip(_slices(s.param, s.sizes, s.gap), s.grads, s.decay)
    out = [_exact_tensor(s, i, *x) for i, x in enumerate(parts)]
    if s.bits == 8:
        p, m, v = zip(*out)
        return p, None if s.copy is None else p, m, v
    p, m, v = torch.zeros(3, s.param.numel(), dtype=torch.float64, device=DEV)
    for flat, new in zip((p, m, v), zip(*out)):
        for to, x in zip(_slices(flat, s.sizes, s.gap), new):
            to.copy_(x)
    return p, None if s.copy is None else p, m, v


def _exact_tensor(s, i, param, grad, decay):
    n = param.numel()
    if s.bits == 32:
        m0, v0 = (_slices(x, s.sizes, s.gap)[i].double() for x in (s.m, s.v))
    else:
        at = torch.arange(n, device=DEV) // BLOCK
        m0, r0 = (code.double() * scale.double()[at]
                  for code, scale in (_views(x[i], n) for x in (s.m, s.v)))
        v0 = r0 ** 2
    g = grad.double() * (1.0 if s.scaled is None else s.scaled.double())
    m1, v1 = torch.lerp(g, m0, B1), torch.lerp(g * g, v0, B2)
    mhat, vhat = m1 / (1 - B1 ** STEP), v1 / (1 - B2 ** STEP)
    p = param.double() * (1 - LR * decay) - LR * mhat / (vhat ** 0.5 + ADAM_EPS)
    if s.bits == 32:
        return p, m1, v1
    h = _hashed(i, n)
    return p, _exact_eight(m1, h >> 16, 0.0), _exact_eight(v1 ** 0.5, h & 0xFFFF, 2.0 ** -9)


def _exact_eight(x, bits, least):
    """(numbers in units of the scales, scales): x rounded to 4 significant bits, or to
    multiples of 2^-9, upwards where what is cut off and the random bits make a whole."""
    n, blocks = x.numel(), -(-x.numel() // BLOCK)
    top = torch.zeros(blocks * BLOCK, dtype=torch.float64, device=DEV)
    top[:n] = x.abs()
    scale = top.view(blocks, BLOCK).max(1).values.div(448).clamp(min=2.0 ** -100)
    y = x / scale.repeat_interleave(BLOCK)[:n]
    unit = torch.exp2((torch.frexp(y)[1] - 4).clamp(min=-9).double())
    z = torch.floor(y.abs() / unit + (bits * 16 + 8).double() / 2 ** 20) * unit
    z = torch.where(y != 0, z.clamp(min=least, max=448.0), z)
    return torch.copysign(z, y), scale
