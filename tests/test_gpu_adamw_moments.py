"""8-bit second moments over many steps: how fast they decay, and which random bits round them.

Rates.  A root r = sqrt(v) without gradients becomes r sqrt(beta2) per step, and rounding with the probability of the remainder leaves its
mean there: after N steps the mean over elements that began at r is r beta2^(N/2).  It may be off by
  - fp32: v's rounding (2^-25 of the root) and the hardware root's (2^-23), N times;
  - chance: N n roundings with probability p <= 16 (1 - beta2)/2 of moving by a code, which is at most r/8: 6 standard deviations of the mean are
    6 r/8 sqrt(N p / n);
  - where 1 - beta2 >= 2^-10, 1/32 of the decay.
"""
import numpy as np
import pytest

from oracle import router as o

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
b = pytest.importorskip("paper_2603_06626_amd.binding")

DEV = "cuda:0"


def states(n, codes):
    z = lambda m, dtype=torch.uint8: torch.zeros(m, dtype=dtype, device=DEV)  # noqa: E731
    v, grad = codes.clone(), z(n, torch.float32)
    kw = dict(m_exp=[z(n // 32)], v_exp=[torch.full((n // 32,), 120, dtype=torch.uint8, device=DEV)])
    return b.AdamWTensors([z(n, torch.float32)], [grad], [z(n)], [v], **kw), v, kw["v_exp"][0], grad


@pytest.mark.parametrize("beta2", [0.99, 0.999, 0.9991, 0.9995, 0.9999, 0.99999])
def test_roots_decay_at_their_rate(beta2):
    n, N = 1 << 24, 40
    codes = torch.randint(112, 127, (n,), dtype=torch.uint8, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    codes.view(-1, 32)[:, 0] = 126             # (its 448 fixes the block's exponent while no more than half of it decays)
    t, v, exps, _ = states(n, codes)
    for step in range(1, N + 1):
        b.grouter_adamw(t, b.grouter_adamw_hyper(lr=1e-3, beta1=0.9, beta2=beta2, eps=1e-8, weight_decay=0.0, step=step, seed=1000 * step + 7))
    assert (exps == 120).all()
    value = torch.from_numpy(o.E4M3[:127]).to(DEV)
    now = value[v.long()]
    for code in range(112, 127):
        mine = codes == code
        count, r = int(mine.sum()), o.E4M3[code]
        want = r * float(np.float32(beta2)) ** (N / 2)
        chance = 6 * r / 8 * (N * 8 * (1 - beta2) / count) ** 0.5
        coarse = (r - want) / 32 if np.float32(1 - beta2) >= 2.0 ** -10 else 0.0
        got = now[mine].mean().item()
        assert abs(got - want) <= N * (2.0 ** -25 + 2.0 ** -23) * r + chance + coarse, (code, got, want, r)


@pytest.mark.parametrize("beta2", [0.999, 0.9999, 0.999999])
def test_codes_follow_from_the_bits(beta2):
    """Moments with every product and sum rounded to fp32, roots rounded to nearest: every code follows from the element's random bits."""
    n, f = 1 << 20, np.float32
    rng = np.random.default_rng(5)
    start = torch.from_numpy(rng.integers(8, 127, n).astype(np.uint8)).to(DEV)
    t, v, exps, grad = states(n, start)
    cv, ev = start.cpu().numpy(), exps.cpu().numpy().astype(np.int64)
    for step in range(1, 4):
        g = (rng.normal(size=n) * 2.0).astype(f)
        grad.copy_(torch.from_numpy(g))
        b.grouter_adamw(t, b.grouter_adamw_hyper(lr=1e-3, beta1=0.9, beta2=beta2, eps=1e-8, weight_decay=0.0, step=step, seed=step))
        old = o.E4M3.astype(f)[cv] * np.repeat(2.0 ** (ev - 127.0), 32).astype(f)
        fv = (old * old) * f(beta2) + (g * g) * f(1 - beta2)
        root = np.sqrt(fv.astype(np.float64)).astype(f)
        ev = o.shared_exponents(np.sqrt(fv.astype(np.float64)))
        up = o.root_bits(o.noise(np.arange(n, dtype=np.uint64), step), beta2)
        y = root * np.repeat(2.0 ** (127.0 - ev), 32).astype(f)
        small = np.floor(y * f(512) + up.astype(f) * f(2.0 ** -20)).astype(np.int64)
        cv = np.minimum(np.where(y < 2.0 ** -6, small, ((y.view(np.uint32).astype(np.int64) + up) >> 20) - 960), 126)
        cv = np.where((y > 0) & (cv < 1), 1, cv).astype(np.uint8)
        assert np.array_equal(exps.cpu().numpy().astype(np.int64), ev) and np.array_equal(v.cpu().numpy(), cv), step
