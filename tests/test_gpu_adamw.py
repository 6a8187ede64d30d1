"""ml2_grad_norm and ml2_adamw against their formulas in 64 bits, within the tolerances that
tests/trainutil.py derives."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402
from tests import trainutil as t  # noqa: E402
from tests.trainutil import TYPES, U, wide  # noqa: E402

DEV = "cuda:0"
HYPER = dict(lr=1e-3, b1=0.9, b2=0.999, eps=1e-8)


def _spread(sizes, dtype, values, gap):
    """Tensors of these values, `gap` elements apart in one buffer, and the buffer."""
    flat = torch.full((sum(sizes) + gap * (len(sizes) + 1),), 7.0, dtype=dtype)
    out, at = [], gap
    for n in sizes:
        out.append((at, n))
        at += n + gap
    for (a, n), v in zip(out, values):
        flat[a: a + n] = torch.from_numpy(np.asarray(v)).to(dtype)
    flat = flat.to(DEV)
    return [flat[a: a + n] for a, n in out], flat


class Case:
    """Tensors with states, and what a step makes of them in 64 bits."""

    def __init__(self, sizes, P, G, bits, gap=0, copy=False, decay=0.1, factor=None, step=3,
                 beside=False, seed=5, rng_seed=0):
        rng = np.random.default_rng(rng_seed + sum(sizes) + len(sizes))
        self.sizes, self.P, self.G, self.bits, self.step, self.seed = sizes, P, G, bits, step, seed
        rand = lambda size: [size * rng.standard_normal(n) * np.exp(rng.standard_normal(n))  # noqa: E731
                             for n in sizes]
        self.p, self.pbuf = _spread(sizes, P, rand(0.02), gap)
        self.g, _ = _spread(sizes, G, rand(0.01), gap)
        m, r = rand(0.003), [np.abs(x) for x in rand(0.01)]
        self.decay = decay if hasattr(decay, "__len__") else [decay] * len(sizes)
        self.copies = _spread(sizes, G, [np.zeros(n) for n in sizes], gap)[0] if copy else None
        if bits == 32:
            self.m, self.mbuf = _spread(sizes, torch.float32, m, gap)
            self.v, _ = _spread(sizes, torch.float32, [x * x for x in r], gap)
        else:
            self.m = [t.encode_state(x).to(DEV) for x in m]
            self.v = [t.encode_state(x).to(DEV) for x in r]
        self.factor = None if factor is None else torch.tensor([factor], device=DEV)
        self.old = [[x.clone() for x in xs] for xs in (self.p, self.m, self.v)]
        out = None
        if beside:
            out = [[torch.full_like(x, 3) for x in xs] for xs in (self.p, self.m, self.v)]
        self.plan = ml2.AdamW(self.p, self.g, bits, self.m, self.v, self.copies, self.decay,
                              (HYPER["b1"], HYPER["b2"]), HYPER["eps"], seed, out)
        self.results = out or [self.p, self.m, self.v]

    def run(self, **more):
        self.plan.run(more.pop("lr", HYPER["lr"]), more.pop("step", self.step), self.factor, **more)
        torch.cuda.synchronize()

    def check(self):
        f = 1.0 if self.factor is None else float(self.factor)
        for i, n in enumerate(self.sizes):
            if n == 0:
                continue
            p, g = wide(self.old[0][i]), wide(self.g[i])
            if self.bits == 32:
                m, v = wide(self.old[1][i]), wide(self.old[2][i])
            else:
                m = t.decoded(self.old[1][i], n)
                v = np.square(t.decoded(self.old[2][i], n))
            new = t.adamw(p, g, m, v, decay=self.decay[i], step=self.step, factor=f, **HYPER)
            ptol, mtol, vtol = t.adamw_tolerance(p, g, m, v, HYPER["lr"], HYPER["b1"], HYPER["b2"],
                                                 self.decay[i], f, new, self.P)
            got = wide(self.results[0][i])
            assert np.all(np.abs(got - new[0]) <= ptol), (i, np.max(np.abs(got - new[0]) - ptol))
            if self.copies is not None:
                ctol = ptol + t.ROUND[self.G] * np.abs(new[0]) * 1.01 + t.TINY[self.G]
                assert np.all(np.abs(wide(self.copies[i]) - new[0]) <= ctol)
            if self.bits == 32:
                assert np.all(np.abs(wide(self.results[1][i]) - new[1]) <= mtol)
                assert np.all(np.abs(wide(self.results[2][i]) - new[2]) <= vtol)
            else:
                h = t.hashed(self.seed, self.step, i, np.arange(n))
                # m's error is relative to its two parts, which may cancel
                ok = np.abs(new[1]) > 0.01 * (0.9 * np.abs(m) + 0.1 * np.abs(g * f))
                t.check_state(self.results[1][i], n, new[1], h >> 16, 0, 500 * U, ok)
                t.check_state(self.results[2][i], n, np.sqrt(new[2]), h & 0xFFFF, 1, 10 * U,
                              np.ones(n, bool))


SIZES = [1, 2, 3, 5, 63, 64, 255, 256, 257, 511, 513, 1000, 2047, 2048, 2049, 4097, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("P", TYPES)
@pytest.mark.parametrize("G", TYPES)
def test_types_and_sizes(bits, P, G):
    print(f"[adamw] {bits} bits {P} {G}", flush=True)
    for gap in (0, 1, 8):
        c = Case(SIZES, P, G, bits, gap, copy=gap == 1, factor=0.37 if gap else None)
        before = c.pbuf.clone()
        c.run()
        c.check()
        if gap:
            assert torch.all(c.pbuf[:gap] == before[:gap]) and torch.all(c.pbuf[-gap:] == 7.0)
            assert torch.all(c.pbuf[gap + 1: 2 * gap + 1] == 7.0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 47, 48, 49, 97, 200])
def test_many_tensors(bits, count):
    """Tables of tensors that fill a launch, and more; some tensors are empty."""
    rng = np.random.default_rng(count)
    sizes = [int(x) for x in rng.integers(0, 6000, count)]
    sizes[0] = 300
    sizes[count // 2] = 0 if count > 1 else 300
    c = Case(sizes, torch.float32, torch.bfloat16, bits, copy=True,
             decay=[0.1 * (i % 3) for i in range(count)])
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("step", [1, 2, 1000, 2 ** 31 - 1])
def test_steps_beside(bits, step):
    """The old state stays as it was; accept() goes on from the new one."""
    c = Case([1000, 1, 4099], torch.float32, torch.float32, bits, step=step, beside=True)
    c.run()
    c.check()
    for have, want in zip((c.p, c.m, c.v), c.old):
        assert all(torch.equal(a, b) for a, b in zip(have, want))
    first = [[x.clone() for x in xs] for xs in c.results]
    c.run()  # again from the same state: the same bits
    for a, b in zip(first, c.results):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    c.plan.accept()
    c.run(step=5)
    d = Case([1000, 1, 4099], torch.float32, torch.float32, bits, step=step)
    d.run()
    d.run(step=5)
    for have, want in zip((c.p, c.m, c.v), (d.p, d.m, d.v)):
        if bits == 8:  # what lies behind a state's elements is nobody's
            have, want = ([torch.cat(ml2_parts(x, n)) for x, n in zip(xs, c.sizes)]
                          for xs in (have, want)) if have is not c.p else (have, want)
        assert all(torch.equal(a, b) for a, b in zip(have, want))


def ml2_parts(state, n):
    codes, scales = ml2.adamw_state_parts(state, n)
    return codes.view(torch.uint8), scales.view(torch.uint8)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("beside", [False, True])
@pytest.mark.parametrize("factor", [float("nan"), float("inf"), -float("inf")])
def test_a_factor_that_is_not_finite_changes_nothing(bits, beside, factor):
    c = Case([1000, 257], torch.bfloat16, torch.float32, bits, copy=True, factor=factor,
             beside=beside)
    c.run()
    for have, want in zip(c.results, c.old):
        for i, (a, b) in enumerate(zip(have, want)):
            if bits == 8 and have is not c.results[0]:
                a, b = (torch.cat(ml2_parts(x, c.sizes[i])) for x in (a, b))
            assert torch.equal(a, b)
    for a, b in zip(c.copies, c.old[0]):
        assert torch.equal(a, b.float())


def test_device_rates_give_the_same_bits():
    """Learning rate and step taken on the device."""
    a, b = (Case([3000, 70], torch.float32, torch.float32, 32, step=7) for _ in range(2))
    a.run()
    b.run(lr=torch.tensor([HYPER["lr"]], device=DEV),
          step=torch.tensor([7], dtype=torch.int32, device=DEV))
    # lr is a float32 on the device: its rate may differ in the last places
    for x, y in zip((*a.m, *a.v), (*b.m, *b.v)):
        assert torch.equal(x, y)
    b.check()
    c = Case([3000, 70], torch.float32, torch.float32, 32, step=1)
    c.run(step=torch.tensor([-4], dtype=torch.int32, device=DEV))  # taken as 1
    c.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_nan_and_infinite_gradients(bits):
    """In 32 bits an element's own state is lost, in 8 bits its block's."""
    n = 1000
    a, b = (Case([n], torch.float32, torch.float32, bits) for _ in range(2))
    b.g[0][300], b.g[0][700] = float("nan"), float("inf")
    a.run()
    b.run()
    lost = np.zeros(n, bool)
    lost[[300, 700]] = True
    states = [wide(x[0]) if bits == 32 else t.decoded(x[0], n) for x in (a.m, b.m, a.v, b.v)]
    p = wide(a.p[0]), wide(b.p[0])
    assert np.array_equal(p[0][~lost], p[1][~lost]) and not np.isfinite(p[1][lost]).any()
    if bits == 8:
        lost = np.repeat([False, True, True, False], 256)[:n]
        assert np.isnan(states[1][lost]).all() and np.isnan(states[3][lost]).all()
    for x, y in (states[:2], states[2:]):
        assert np.array_equal(x[~lost], y[~lost]) and not np.isfinite(y[lost]).any()


def test_extreme_sizes_of_gradients():
    """Squares that leave float32 at both ends, zeros, and blocks of 8-bit states of them."""
    n = 1024
    for bits in (32, 8):
        c = Case([n], torch.float32, torch.float32, bits)
        for x in (c.m[0], c.v[0]):
            x.zero_()
        c.g[0][:256] = 0.0
        c.g[0][256:512] = 1e-30
        c.g[0][512:768] = 1e15
        c.g[0][768:] = -1e-9
        c.old[1][0].zero_()
        c.old[2][0].zero_()
        c.run(step=1)
        p, old = wide(c.p[0]), wide(c.old[0][0])
        kept = old * (1 - 1e-3 * 0.1)
        # no gradient: decay alone; 1e-30: far below eps; 1e15: one learning rate
        assert np.allclose(p[:512], kept[:512], rtol=1e-6, atol=1e-24)
        assert np.allclose(p[512:768], kept[512:768] - 1e-3, rtol=1e-5, atol=1e-9)
        up = p[768:] - kept[768:]
        assert np.all((up > 0) & (up < 1.01e-3))
        m = wide(c.m[0]) if bits == 32 else t.decoded(c.m[0], n)
        v = wide(c.v[0]) if bits == 32 else np.square(t.decoded(c.v[0], n))
        assert np.all(m[:256] == 0) and np.all(v[:256] == 0)
        # equal elements are the top of their block: no rounding but float32's
        assert np.allclose(m[512:768], 1e14, rtol=1e-6) and np.allclose(v[512:768], 1e27, rtol=1e-5)


@pytest.mark.parametrize("step", [1, 7])
def test_states_in_8_bits_code_for_code(step):
    """The documented float32 arithmetic, worked out by numpy.  A size is other than numpy's only
    where a root or a block's 1 / scale is the number next to the nearest: by at most 2 of its last
    bits, so that its code is another one with a chance of 2 in 2^20 (the bits that decide are
    spread evenly over them): 0.5 of the 2^18 elements on average, were every one of them off.
    Fewer than 8 differ, by one code, but for a chance of 1e-7."""
    n, f32 = 1 << 18, np.float32
    c = Case([n], torch.float32, torch.float32, 8, step=step)
    c.run()
    b1, b2, a1, a2 = (f32(x) for x in (0.9, 0.999, 1 - 0.9, 1 - 0.999))
    g = c.g[0].cpu().numpy()
    m, r = (t.values(codes).astype(f32) * np.repeat(scale.astype(f32), t.BLOCK)[:n]
            for codes, scale in (t.split(x[0], n) for x in c.old[1:]))
    m = m * b1 + g * a1
    r = np.sqrt(r * r * b2 + g * a2 * g)
    h = t.hashed(c.seed, step, 0, np.arange(n))
    for x, state, bits, least in ((m, c.m[0], h >> 16, 0), (r, c.v[0], h & 0xFFFF, 1)):
        assert x.dtype == f32
        scale = np.maximum(np.abs(x).reshape(-1, t.BLOCK).max(1) * f32(1 / 448), f32(2.0 ** -100))
        size = np.abs(x) * np.repeat(f32(1) / scale, t.BLOCK)
        want = (size * f32(2.0 ** -120)).view(np.uint32).astype(np.int64) + bits * 16 + 8 >> 20
        want = np.minimum(np.maximum(want, least * (x != 0)), 126)
        codes, got_scale = t.split(state, n)
        assert np.all(np.abs(got_scale - scale) <= 4 * U * scale)
        off = np.abs((codes & 127).astype(np.int64) - want)
        assert off.max() <= 1 and off.sum() < 8
        assert np.array_equal(codes >= 128, np.signbit(x))


def test_slow_averages_move_in_8_bits():
    """3,000 steps of one gradient a tensor's element: both averages arrive at it.  The mean of
    4,096 unbiased chains is off by far less than the 5 % asked for; rounding to the nearest would
    leave v where a step changes it by less than half a code, at a fiftieth of g^2."""
    n = 4096
    g = torch.from_numpy(np.random.default_rng(2).uniform(0.5, 2.0, n)).float().to(DEV)
    p = torch.zeros(n, device=DEV)
    plan = ml2.AdamW([p], [g], 8, weight_decay=0.0)
    for step in range(1, 3001):
        plan.run(0.0, step)
    torch.cuda.synchronize()
    m, r = t.decoded(plan.m[0], n), t.decoded(plan.v[0], n)
    assert abs((m / wide(g)).mean() - 1) < 0.05
    # the mean of squares lies above the square of the mean by the roundings' spread
    share = np.square(r).mean() / np.square(wide(g)).mean()
    assert 0.9 < share < 1.15


@pytest.mark.parametrize("n", [(1 << 32) + 1000])
def test_indices_beyond_32_bits(n):
    """8-bit states and 16-bit parameters of more than 2^32 elements: the ends."""
    print("[adamw] 2^32 + 1000 elements", flush=True)
    free, _ = torch.cuda.mem_get_info()
    if free < 30 << 30:
        pytest.skip("30 GiB of device memory are needed")
    p = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    m, v = (torch.zeros(ml2.ml2_adamw_state_bytes(8, n), dtype=torch.uint8, device=DEV)
            for _ in range(2))
    rng = np.random.default_rng(1)
    tail = torch.from_numpy(rng.standard_normal(3048)).bfloat16()
    g[-3048:] = tail.to(DEV)
    g[:3048] = tail.to(DEV)
    norm = ml2.GradNorm([g]).run()[0]
    plan = ml2.AdamW([p], [g], 8, [m], [v], weight_decay=0.0, seed=9)
    plan.run(1e-3, 2)
    torch.cuda.synchronize()
    want = np.sqrt(2 * np.square(wide(tail)).sum())
    assert abs(float(norm) - want) <= 2 * U * want
    b1, b2 = 0.9, 0.999
    blocks = -(-n // 256)
    for first in (0, n - 3048):
        at = np.arange(first, first + 3048)
        d = wide(tail)
        zeros = np.zeros(3048)
        new = t.adamw(zeros, d, zeros, zeros, 1e-3, b1, b2, 1e-8, 0.0, 2)
        tol = t.adamw_tolerance(zeros, d, zeros, zeros, 1e-3, b1, b2, 0.0, 1.0, new,
                                torch.bfloat16)[0]
        assert np.all(np.abs(wide(p[first: first + 3048]) - new[0]) <= tol)
        lo = (at >> 32) == 0
        h = np.concatenate([t.hashed(9, 2, 0, at[lo]), t.hashed(9, 2, 0, at[~lo])])
        s0, skip = first // 256, first % 256
        for state, value, bits, least in ((m, new[1], h >> 16, 0),
                                          (v, np.sqrt(new[2]), h & 0xFFFF, 1)):
            # the blocks that begin inside the piece, as a state of their own
            a = (256 - skip) % 256
            count = 3048 - a
            k0 = s0 + (1 if a else 0)
            k1 = min(blocks, k0 + -(-count // 256))
            part = torch.cat([state[first + a: first + 3048],
                              torch.zeros(-count % 256, dtype=torch.uint8, device=DEV),
                              state[blocks * 256 + 4 * k0: blocks * 256 + 4 * k1]])
            if first == 0:  # the last block goes on behind the piece, with zeros
                pass
            t.check_state(part, count, value[a:], bits[a:], least, 500 * U, np.ones(count, bool))
    del p, g, m, v


# ---- norms -----------------------------------------------------------------------------

def _norm_case(sizes, dtype, gap, scale, max_norm, size=1.0):
    rng = np.random.default_rng(sum(sizes) + len(sizes))
    grads, _ = _spread(sizes, dtype, [size * rng.standard_normal(n) for n in sizes], gap)
    step = torch.tensor([4], dtype=torch.int32, device=DEV)
    norm, factor = ml2.GradNorm(grads, max_norm, scale, step).run()
    torch.cuda.synchronize()
    want = scale * np.sqrt(sum(np.square(wide(g)).sum() for g in grads))
    f = scale * (min(1.0, max_norm / want) if want > 0 else 1.0)
    # one rounding to float32 each, and those of the scale and the limit on their way here
    assert abs(float(norm) - want) <= 3 * U * want
    assert abs(float(factor) - f) <= 4 * U * f
    assert int(step) == 5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [[1], [0, 3], [50000], [65536], [65537], [131072], [131073], [1000] * 16, [1000] * 17,
                                   [1] * 64, [1] * 65,
                                   [7] * 128, [9] * 129, [333] * 400, [1 << 22, 5, 100001],
                                   [40000001]])
def test_norms(dtype, sizes):
    for gap in (0, 1):
        for scale, limit in ((1.0, 1.0), (0.25, float("inf")), (2.0, 1e9)):
            _norm_case(sizes, dtype, gap, scale, limit)


def test_norms_of_extreme_values():
    _norm_case([5000], torch.float32, 0, 1.0, 1.0, size=1e30)   # squares beyond float32
    _norm_case([5000], torch.float32, 0, 1.0, 1.0, size=1e-30)
    _norm_case([300000], torch.bfloat16, 0, 1.0, 1.0, size=1e34)
    z = torch.zeros(100, device=DEV)
    norm, factor = ml2.GradNorm([z], 0.5).run()
    assert float(norm) == 0.0 and float(factor) == 1.0


@pytest.mark.parametrize("n", [100, 300000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite(n, bad):
    g = torch.ones(n, device=DEV)
    g[n // 2] = bad
    step = torch.tensor([4], dtype=torch.int32, device=DEV)
    norm, factor = ml2.GradNorm([g], 1.0, step=step).run()
    torch.cuda.synchronize()
    assert not np.isfinite(float(norm)) and np.isnan(float(factor)) and int(step) == 4
    g.fill_(3e38)  # finite elements, a norm beyond float32
    norm, factor = ml2.GradNorm([g], 1.0, step=step).run()
    assert np.isinf(float(norm)) and np.isnan(float(factor)) and int(step) == 4


def test_nothing_to_sum_or_step():
    z = torch.zeros(0, device=DEV)
    norm, factor = ml2.GradNorm([z], 1.0).run()
    assert float(norm) == 0.0 and float(factor) == 1.0
    ml2.AdamW([z], [z.clone()]).run(1e-3, 1)
    ml2.AdamW([z], [z.clone()], 8).run(1e-3, 1)
    ml2.ml2_adamw(torch.float32, torch.float32, 32, None, 0,
                  ml2.ml2_adamw_options(1e-3, 0.9, 0.999, 1e-8, 1, None, None, None, 0))
    out = (ctypes.c_size_t * 1)()
    assert ml2.lib().ml2_grad_norm_workspace_bytes(None, 0, out) == 0
    torch.cuda.synchronize()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_follows_its_counter(bits):
    """Norm, factor, counter and step in one graph: each replay is the eager step with the next
    number, and one whose gradients are not finite leaves parameters, states and counter."""
    sizes = [3000, 70001, 5]

    def program():
        c = Case(sizes, torch.float32, torch.bfloat16, bits, copy=True)
        c.count = torch.zeros(1, dtype=torch.int32, device=DEV)
        c.rate = torch.tensor([1e-3], device=DEV)
        c.norm = ml2.GradNorm(c.g, 0.5, step=c.count)
        return c

    def step(c):
        _, factor = c.norm.run()
        c.plan.run(c.rate, c.count, factor)

    a, b = program(), program()
    step(a)
    step(b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(a)
    for turn in range(5):
        grads = [torch.randn(n, device=DEV).bfloat16() * 0.01 for n in sizes]
        if turn == 2:
            grads[1][500] = float("inf")
        for c in (a, b):
            c.rate.fill_(1e-3 / (turn + 1))
            for to, x in zip(c.g, grads):
                to.copy_(x)
        g.replay()
        step(b)
        torch.cuda.synchronize()
        assert int(a.count) == int(b.count) == (turn + 2 if turn < 2 else turn + 1)
        for x, y in zip((*a.p, *a.copies), (*b.p, *b.copies)):
            assert torch.equal(x, y)
        for x, y in zip((*a.m, *a.v), (*b.m, *b.v)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("bits", [32, 8])
def test_other_gradients(bits):
    """take(): the next call is that of objects made with those gradients."""
    a = Case([1000, 3, 700], torch.float32, torch.bfloat16, bits, factor=0.5)
    b = Case([1000, 3, 700], torch.float32, torch.bfloat16, bits, factor=0.5)
    fresh = [torch.randn(n, device=DEV).bfloat16() for n in a.sizes]
    norm = ml2.GradNorm(a.g, 1.0)
    for to, x in zip(b.g, fresh):
        to.copy_(x)
    norm.take(fresh)
    a.plan.take(fresh)
    a.run()
    b.run()
    for have, want in zip((a.p, a.m, a.v), (b.p, b.m, b.v)):
        assert all(torch.equal(x, y) for x, y in zip(have, want))
    assert torch.equal(norm.run()[0], ml2.GradNorm(b.g, 1.0).run()[0])
    for bad in (fresh[:2], [fresh[0], fresh[1], fresh[2][:-1]], [x.float() for x in fresh],
                [None] * 3):
        for taker in (norm, a.plan):
            with pytest.raises(ValueError):
                taker.take(bad)


@pytest.mark.parametrize("which", ["lr", "step", "factor"])
def test_rates_of_another_device_are_refused(which):
    """(here: seen so)"""
    class Far(torch.Tensor):
        def get_device(self):
            return torch.cuda.current_device() + 1

    args = dict(lr=torch.ones(1, device=DEV), step=torch.ones(1, dtype=torch.int32, device=DEV),
                factor=torch.ones(1, device=DEV))
    c = Case([5], torch.float32, torch.float32, 32)
    c.plan.run(**args)
    args[which] = args[which].as_subclass(Far)
    with pytest.raises(ValueError, match="current"):
        c.plan.run(**args)


@pytest.mark.parametrize("bits", [32, 8])
def test_rates_of_numpy(bits):
    """numpy's numbers are numbers: the same bits as Python's."""
    a, b = (Case([3000, 70], torch.float32, torch.float32, bits, step=7) for _ in range(2))
    a.run(lr=2.0 ** -10, step=7)
    b.run(lr=np.float32(2.0 ** -10), step=np.int64(7))
    for x, y in zip((*a.p, *a.m, *a.v), (*b.p, *b.m, *b.v)):
        assert torch.equal(x, y)
    for bad in (7.0, np.float64(7), "7"):
        with pytest.raises((ValueError, AttributeError)):
            a.plan.run(2.0 ** -10, bad)


def test_a_step_without_its_rates_is_refused():
    """None is not the rate or the step of the call before."""
    c = Case([50], torch.float32, torch.float32, 32)
    c.run()
    kept = c.p[0].clone()
    for lr, step in ((None, 3), (1e-3, None), (None, None)):
        with pytest.raises(ValueError, match="given"):
            c.plan.run(lr, step)
    torch.cuda.synchronize()
    assert torch.equal(c.p[0], kept)


def _state_bytes(c):
    """What a step has left of every tensor, without the bytes behind an 8-bit state's elements."""
    if c.bits == 32:
        return [*c.p, *c.m, *c.v]
    return c.p + [torch.cat(ml2_parts(x, n)) for xs in (c.m, c.v) for x, n in zip(xs, c.sizes)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("P,G", [(torch.float32, torch.float32), (torch.bfloat16, torch.float16)])
@pytest.mark.parametrize("step", [1, 7, 1000, 2 ** 31 - 1])
def test_device_and_host_rates_agree_in_every_bit(bits, P, G, step):
    """Parameters, and for 8 bits codes and scales, of a step whose rate and number lie on the device
    are those of the same step from the host: float32 holds the rate, and the two rates are worked
    out in float64 on both sides, so that they round to other float32 numbers only where the
    functions' last places decide, with a chance of some 2^-28.  A number off by one gives other
    parameters (but for steps so late that the corrections are 1) and other codes."""
    sizes, lr = [3000, 70, 4097], 2.0 ** -10

    def stepped(**rates):
        c = Case(sizes, P, G, bits, step=step)
        c.run(**rates)
        return _state_bytes(c)

    def device(n):
        return torch.tensor([n], dtype=torch.int32, device=DEV)

    want = stepped(lr=lr, step=step)
    rate = torch.tensor([lr], device=DEV)
    for rates in (dict(lr=rate, step=device(step)), dict(lr=rate, step=step),
                  dict(lr=lr, step=device(step))):
        assert all(torch.equal(a, b) for a, b in zip(stepped(**rates), want)), rates.keys()
    other = stepped(lr=rate, step=device(step - 1 if step > 1 else 2))
    if step < 1000:
        assert not torch.equal(other[0], want[0])
    if bits == 8:
        assert not torch.equal(other[3], want[3]) and not torch.equal(other[6], want[6])
    assert not torch.equal(stepped(lr=2 * rate, step=device(step))[0], want[0])


@pytest.mark.parametrize("step", [3, 1000])
def test_states_in_8_bits_by_the_devices_step(step):
    """Parameters, codes and scales against 64 bits, rate and number on the device."""
    c = Case([3000, 70, 4097], torch.float32, torch.float32, 8, step=step)
    c.run(lr=torch.tensor([HYPER["lr"]], device=DEV),
          step=torch.tensor([step], dtype=torch.int32, device=DEV))
    c.check()


@pytest.mark.parametrize("seed", [0, (3 << 32) | 5, 5 << 32, 2 ** 64 - 1])
def test_seeds_of_64_bits(seed):
    """Both words of the seed are in the hash."""
    c, low = (Case([3000, 70], torch.float32, torch.float32, 8, seed=s) for s in (seed, seed & t.LOW))
    c.run()
    low.run()
    c.check()
    assert torch.equal(c.m[0], low.m[0]) == (seed < 1 << 32)
