"""AdamW over lists of tensors against the 64-bit oracle.

Tolerances.  m and v: two products and a sum, at most 3 roundings of 2^-24 each, of terms that may cancel in m.  w: the step is
lr m / (sqrt(v) + eps), whose relative error is below 1e-6 (m's roundings, hardware root and reciprocal of 1 unit each), plus one rounding
of the result.  Codes and bf16 parameters that are rounded by random bits lie next to the exact value; which of the two neighbours it is
follows from the bits wherever the exact remainder is not within 1e-3 of the border.
"""
import numpy as np
import pytest

from oracle import router as o

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
b = pytest.importorskip("paper_2603_06626_amd.binding")

DEV = "cuda:0"
SIZES = [1, 0, 7, 8, 9, 31, 32, 33, 64, 255, 2048, 8191, 8192, 8193, 20003]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


def padded(n, dtype, fill):
    """A tensor of n elements with guards on both sides, 16-byte aligned."""
    whole = torch.full((n + 128,), fill, dtype=dtype, device=DEV)
    return whole[64:64 + n], whole


class Case:
    def __init__(self, sizes, kind, grad, bits, seed=0, fill=0):
        rng = np.random.default_rng(seed)
        self.sizes, self.kind, self.bits = sizes, kind, bits
        self.whole = []

        def make(dtype, values):
            out = []
            for n, v in zip(sizes, values):
                t, w = padded(n, dtype, 3)
                t.copy_(torch.from_numpy(np.asarray(v)).to(DEV).to(dtype))
                self.whole.append((w, n))
                out.append(t)
            return out

        values = [rng.normal(size=n) for n in sizes]
        self.param = make(torch.float32 if kind == "fp32" else torch.bfloat16, values)
        self.master = make(torch.float32, values) if kind == "master" else None
        self.grad = make(torch.float32 if grad == "fp32" else torch.bfloat16, [rng.normal(size=n) * np.exp(rng.normal(size=n) * 3) * 1e-2 for n in sizes])
        self.m_exp = self.v_exp = None
        if bits == 32:
            self.m = make(torch.float32, [rng.normal(size=n) * 1e-2 for n in sizes])
            self.v = make(torch.float32, [rng.normal(size=n) ** 2 * 1e-4 for n in sizes])
        else:
            self.m = make(torch.uint8, [rng.integers(0, 127, size=n) + 128 * rng.integers(0, 2, size=n) for n in sizes])
            self.v = make(torch.uint8, [rng.integers(0, 127, size=n) for n in sizes])
            self.m_exp, self.v_exp = ([torch.from_numpy(rng.integers(110, 116, size=-(-n // 32)).astype(np.uint8)).to(DEV) for n in sizes] for _ in range(2))
        self.list = b.AdamWTensors(self.param, self.grad, self.m, self.v, master=self.master, m_exp=self.m_exp, v_exp=self.v_exp)

    def state(self):
        """w, g, m, v of every tensor in 64 bits."""
        out = []
        for i, n in enumerate(self.sizes):
            w = (self.param if self.master is None else self.master)[i].double().cpu().numpy()
            g = self.grad[i].double().cpu().numpy()
            if self.bits == 32:
                m, v = self.m[i].double().cpu().numpy(), self.v[i].double().cpu().numpy()
            else:
                m = o.decode(self.m[i].cpu().numpy(), self.m_exp[i].cpu().numpy())
                v = o.decode(self.v[i].cpu().numpy(), self.v_exp[i].cpu().numpy()) ** 2
            out.append((w, g, m, v))
        return out

    def guards_hold(self):
        return all((w[:64] == 3).all() and (w[64 + n:] == 3).all() for w, n in self.whole)


def expected_up(fraction, bits, width):
    """Whether the upper neighbour is due, and where that is certain."""
    reach = fraction + bits / 2.0 ** width
    return reach >= 1.0, np.abs(reach - 1.0) > 1e-3


def check_codes(codes, exps, x, noise20, least):
    """codes stand for x >= 0, rounded to one of its neighbours by the random bits; exponents are the least that fit."""
    want = o.shared_exponents(x)
    got = exps.astype(np.int64)
    if not np.array_equal(got, want):      # a block whose largest lies within 1e-6 of the border may take the next one
        for i in np.argwhere(got != want)[:, 0]:
            top = x[32 * i:32 * i + 32].max()
            # (a block of zeros has no exponent that matters)
            assert top == 0 or abs(np.log2(top / 448.0) - round(np.log2(top / 448.0))) < 1e-6, (i, top)
    value = np.abs(o.decode(codes, exps))
    low, high = o.neighbours(x, got)
    smallest = np.repeat(2.0 ** (got - 127.0 - 9), 32)[:len(x)]
    assert ((value >= low * (1 - 1e-5) - 1e-30) & (value <= high * (1 + 1e-5) + 1e-30) | (np.abs(x - value) < 1e-5 * x)).all()
    gap = np.where(high > low, high - low, 1.0)
    up, sure = expected_up((x - low) / gap, noise20, 20)
    due = np.where((high > low) & up, high, low)
    if least:
        due = np.where((x > 0) & (due == 0), smallest, due)
    near = np.minimum(np.abs(x - low), np.abs(x - high)) < 1e-5 * x
    assert (np.abs(value - due)[sure & ~near] == 0).all()


def check_step(c, before, step, seed, scale=1.0, hyper=HYPER):
    for i, (w, g, m, v) in enumerate(before):
        rw, rm, rv = o.adamw(w, g, m, v, step=step, grad_scale=scale, **hyper)
        n = len(w)
        noise = o.noise(o.places_of(c.sizes)[i], seed).astype(np.int64)
        move = np.abs(rw - w) + np.abs(rw) * 2.0 ** -24
        if c.kind == "bf16":
            got = c.param[i].double().cpu().numpy()
            unit = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(rw), 1e-300))) - 7)
            assert (np.abs(got - rw) <= unit * (1 + 1e-3)).all()
            low = np.floor(np.abs(rw) / unit)
            up, sure = expected_up(np.abs(rw) / unit - low, noise >> 16, 16)
            assert (np.abs(got) == (low + up) * unit)[sure].all()
        else:
            got = (c.param if c.master is None else c.master)[i].double().cpu().numpy()
            # m's rounding errors are relative to its two terms, which may cancel: 4 * 2^-24 of their sum, over the root
            lr, root = hyper["lr"] / (1 - hyper["beta1"] ** step), np.sqrt(rv / (1 - hyper["beta2"] ** step)) + hyper["eps"]
            terms = hyper["beta1"] * np.abs(m) + (1 - hyper["beta1"]) * np.abs(g * scale)
            assert (np.abs(got - rw) <= 2e-6 * move + 2.0 ** -24 * (np.abs(rw) + np.abs(w)) + lr * 4 * 2.0 ** -24 * terms / root).all()
            if c.master is not None:
                assert torch.equal(c.param[i], c.master[i].bfloat16())
        if c.bits == 32:
            assert (np.abs(c.m[i].double().cpu().numpy() - rm) <= 4 * 2.0 ** -24 * (np.abs(m) + np.abs(g * scale))).all()
            assert (np.abs(c.v[i].double().cpu().numpy() - rv) <= 6 * 2.0 ** -24 * rv + 1e-44).all()
        elif n:
            codes, exps = c.m[i].cpu().numpy(), c.m_exp[i].cpu().numpy()
            check_codes(codes, exps, np.abs(rm), noise >> 12, False)
            sign = (codes & 0x80) != 0
            assert (sign == (rm < 0))[np.abs(rm) > 1e-12].all()
            check_codes(c.v[i].cpu().numpy(), c.v_exp[i].cpu().numpy(), np.sqrt(rv), (noise & 0xfff) * 256 + 128, True)
    assert c.guards_hold()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["fp32", "master", "bf16"])
def test_steps(kind, grad, bits):
    c = Case(SIZES, kind, grad, bits)
    for step, seed in ((1, 5), (2, 6), (1000, 0xffffffff)):
        before = c.state()
        b.grouter_adamw(c.list, b.grouter_adamw_hyper(step=step, seed=seed, **HYPER))
        check_step(c, before, step, seed)


@pytest.mark.parametrize("count", [1, 39, 40, 41, 81, 200])
def test_more_tensors_than_a_launch_takes(count):
    c = Case([(17 * i) % 90 for i in range(count)], "bf16", "bf16", 8, seed=count)
    before = c.state()
    b.grouter_adamw(c.list, b.grouter_adamw_hyper(step=3, seed=9, **HYPER))
    check_step(c, before, 3, 9)


def test_same_call_same_result():
    a, c = Case(SIZES, "bf16", "bf16", 8), Case(SIZES, "bf16", "bf16", 8)
    for x in (a, c):
        b.grouter_adamw(x.list, b.grouter_adamw_hyper(step=1, seed=4, **HYPER))
    assert all(torch.equal(x, y) for i in range(4) for x, y in zip(a.list._held[i], c.list._held[i]))


def test_scale_on_the_device_and_hyper_on_the_device():
    c, e = Case(SIZES, "master", "bf16", 32), Case(SIZES, "master", "bf16", 32)
    before = c.state()
    scale = torch.tensor([0.25], device=DEV)
    h = b.grouter_adamw_hyper(step=7, seed=1, grad_scale=0.5, **HYPER)
    b.grouter_adamw(c.list, h, grad_scale=scale)
    check_step(c, before, 7, 1, scale=0.125)
    b.grouter_adamw(e.list, h.tensor().to(DEV), grad_scale=scale)
    assert all(torch.equal(x, y) for i in (0, 2, 3, 4) for x, y in zip(c.list._held[i], e.list._held[i]))


def test_zero_state_zero_gradient():
    for bits in (32, 8):
        n = 100
        p = torch.ones(n, device=DEV)
        kw = {}
        m, v = (torch.zeros(n, dtype=torch.float32 if bits == 32 else torch.uint8, device=DEV) for _ in range(2))
        if bits == 8:
            kw = dict(m_exp=[torch.zeros(4, dtype=torch.uint8, device=DEV)], v_exp=[torch.zeros(4, dtype=torch.uint8, device=DEV)])
        t = b.AdamWTensors([p], [torch.zeros(n, device=DEV)], [m], [v], **kw)
        b.grouter_adamw(t, b.grouter_adamw_hyper(step=1, **HYPER))
        assert torch.allclose(p, torch.full_like(p, 1 - 1e-3), rtol=1e-6) and (m == 0).all() and (v == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_not_finite_gradients(bad):
    c = Case([100], "fp32", "fp32", 8)
    c.grad[0][40] = bad
    keep = [x.clone() for x in (c.m[0], c.v[0], c.param[0])]
    b.grouter_adamw(c.list, b.grouter_adamw_hyper(step=2, seed=1, **HYPER))
    m = o.decode(c.m[0].cpu().numpy(), c.m_exp[0].cpu().numpy())
    v = o.decode(c.v[0].cpu().numpy(), c.v_exp[0].cpu().numpy())
    for x, e in ((m, c.m_exp), (v, c.v_exp)):
        assert np.isnan(x[32:64]).all() and not np.isnan(np.delete(x, np.arange(32, 64))).any() and e[0][1] == 255
    p = c.param[0].cpu().numpy()
    assert np.isfinite(np.delete(p, 40)).all() and (np.isnan(p[40]) if not np.isfinite(p[40]) else True)
    del keep


def test_small_and_large_moments_keep_their_place():
    """A block with moments 40 binades apart: the small roots stay above 0, the small moments are at most the smallest code."""
    n = 64
    g = torch.zeros(n, device=DEV)
    g[0], g[1:32] = 1.0, 2.0 ** -40
    g[32:] = 2.0 ** -60
    c = b.AdamWTensors([torch.zeros(n, device=DEV)], [g], [torch.zeros(n, dtype=torch.uint8, device=DEV)], [torch.zeros(n, dtype=torch.uint8, device=DEV)],
                       m_exp=[torch.zeros(2, dtype=torch.uint8, device=DEV)], v_exp=[torch.zeros(2, dtype=torch.uint8, device=DEV)])
    for step in range(1, 6):
        b.grouter_adamw(c, b.grouter_adamw_hyper(step=step, seed=step, **HYPER))
    v = c._held[3][0].cpu().numpy()
    assert (v[1:32] == 1).all() and v[0] > 8 and (v[32:] > 8).all()
    p = c._held[0][0].cpu().numpy()
    assert np.isfinite(p).all() and np.abs(p).max() < 0.06       # five steps of at most lr each, and no step divided by eps


def test_moments_in_8_bits_follow_those_in_32():
    """A constant gradient and beta2 = 0.999: rounding to nearest would leave v where it is, random rounding lets it rise as it should.

    The mean of n = 4096 codes after 300 steps differs from the exact root by at most 6 standard errors.  The steps' rounding errors are
    independent with a variance of at most (step/2)^2 each, step = 1/8 of the root at most, and sqrt(v)'s error at one step is carried on
    by less than 1: standard deviation of one element <= sqrt(300) / 16, of the mean / 64, i.e. 6 * 0.017 = 0.10 of the root; the
    convexity of the square, which raises v by the variance of its root each step (at most (1/16)^2), adds at most 300 * 0.0039 / 2 = 0.59
    if it never decayed; it is measured against 1.7 times the root."""
    n, steps, beta2 = 4096, 300, 0.999
    kw = dict(m_exp=[torch.zeros(n // 32, dtype=torch.uint8, device=DEV)], v_exp=[torch.zeros(n // 32, dtype=torch.uint8, device=DEV)])
    t = b.AdamWTensors([torch.zeros(n, device=DEV)], [torch.full((n,), 1e-3, device=DEV)], [torch.zeros(n, dtype=torch.uint8, device=DEV)],
                       [torch.zeros(n, dtype=torch.uint8, device=DEV)], **kw)
    for s in range(1, steps + 1):
        b.grouter_adamw(t, b.grouter_adamw_hyper(lr=1e-3, beta1=0.9, beta2=beta2, eps=1e-8, weight_decay=0.0, step=s, seed=s))
    root = o.decode(t._held[3][0].cpu().numpy(), kw["v_exp"][0].cpu().numpy())
    exact = 1e-3 * np.sqrt(1 - beta2 ** steps)
    assert 0.9 * exact < root.mean() < 1.7 * exact


def codes_in_fp32(x, exps, up, least):
    """The codes of x >= 0 (fp32) as the format defines them, in fp32 and whole numbers."""
    y = x * np.repeat(2.0 ** (127.0 - exps), 32).astype(np.float32)[:len(x)]
    normal = ((y.view(np.uint32).astype(np.int64) + up) >> 20) - 960
    small = np.floor(y * np.float32(512) + up.astype(np.float32) * np.float32(2.0 ** -20)).astype(np.int64)
    code = np.minimum(np.where(y < 2.0 ** -6, small, normal), 126)
    return np.where((y > 0) & (code < least), least, code)


@pytest.mark.parametrize("spread", [0.0, 4.0])
def test_codes_are_those_of_the_formulas_bit_for_bit(spread):
    """Moments in fp32 with every product and sum rounded, roots rounded to nearest: the 8-bit states of millions of elements follow exactly,
    also where gradients span many binades and codes lie in equal steps."""
    n, f = 2_000_032, np.float32
    rng = np.random.default_rng(int(spread))
    kw = dict(m_exp=[torch.zeros(n // 32, dtype=torch.uint8, device=DEV)], v_exp=[torch.zeros(n // 32, dtype=torch.uint8, device=DEV)])
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    grad = torch.zeros(n, device=DEV)
    t = b.AdamWTensors([torch.zeros(n, device=DEV)], [grad], [m], [v], **kw)
    em, ev, cm, cv = np.zeros(n // 32, np.int64), np.zeros(n // 32, np.int64), np.zeros(n, np.int64), np.zeros(n, np.int64)
    for step in range(1, 5):
        g = (rng.normal(size=n) * np.exp(spread * rng.normal(size=n)) * 1e-3).astype(f)
        grad.copy_(torch.from_numpy(g))
        b.grouter_adamw(t, b.grouter_adamw_hyper(step=step, seed=step, **HYPER))
        value = o.E4M3.astype(f)
        sm, sv = (np.repeat(2.0 ** (e - 127.0), 32).astype(f) for e in (em, ev))
        old = value[cv] * sv
        fm = (value[cm] * sm) * f(0.9) + g * f(1 - 0.9)
        fv = (old * old) * f(0.99) + (g * g) * f(1 - 0.99)
        em, ev = o.shared_exponents(np.abs(fm).astype(np.float64)), o.shared_exponents(np.sqrt(fv.astype(np.float64)))
        h = o.noise(np.arange(n, dtype=np.uint64), step).astype(np.int64)
        cm = codes_in_fp32(np.abs(fm), em, h >> 12, 0) + 128 * np.signbit(fm)
        cv = codes_in_fp32(np.sqrt(fv.astype(np.float64)).astype(f), ev, (h & 0xfff) * 256 + 128, 1)
        for got, want in ((kw["m_exp"][0], em), (kw["v_exp"][0], ev), (m, cm), (v, cv)):
            assert np.array_equal(got.cpu().numpy().astype(np.int64), want), step


def test_steps_in_a_graph_replay_with_the_buffers_contents():
    c, e = Case(SIZES, "bf16", "bf16", 8), Case(SIZES, "bf16", "bf16", 8)
    hyper = torch.zeros(48, dtype=torch.uint8, device=DEV)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        b.grouter_adamw(c.list, hyper)
    for step in (1, 2, 3):
        h = b.grouter_adamw_hyper(step=step, seed=100 + step, **HYPER)
        hyper.copy_(h.tensor())
        graph.replay()
        torch.cuda.synchronize()
        b.grouter_adamw(e.list, h)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for i in (0, 2, 3, 5, 6) for x, y in zip(c.list._held[i], e.list._held[i])), step


def test_list_refusals():
    x = lambda n=64, dtype=torch.float32: torch.zeros(n, dtype=dtype, device=DEV)  # noqa: E731
    p, g, m, v = x(), x(), x(), x()
    b.AdamWTensors([p], [g], [m], [v])
    for bad in (lambda: b.AdamWTensors([p], [p], [m], [v]), lambda: b.AdamWTensors([p, p], [g, x()], [m, x()], [v, x()]),
                lambda: b.AdamWTensors([p], [x(63)], [m], [v]), lambda: b.AdamWTensors([p], [g], [x(64, torch.float16)], [v]),
                lambda: b.AdamWTensors([x(64, torch.float16)], [g], [m], [v]), lambda: b.AdamWTensors([p], [g], [m], [v], master=[x()]),
                lambda: b.AdamWTensors([x(65)[1:]], [g], [m], [v]), lambda: b.AdamWTensors([p], [g], [x(64, torch.uint8)], [x(64, torch.uint8)]),
                lambda: b.AdamWTensors([p], [g], [m], [v], m_exp=[x(2, torch.uint8)], v_exp=[x(2, torch.uint8)]),
                lambda: b.AdamWTensors([p, x(64, torch.bfloat16)], [g, x()], [m, x()], [v, x()]), lambda: b.AdamWTensors([p], [g], [x(128)[::2]], [v])):
        with pytest.raises(ValueError):
            bad()
    b.grouter_adamw(b.AdamWTensors([], [], [], []), b.grouter_adamw_hyper(step=1, **HYPER))
