"""Pins of the router's, the balance loss's and AdamW's 64-bit oracle: closed forms, identities and central differences (no GPU)."""
import numpy as np
import pytest

from oracle import router as o

GATINGS = [o.SOFTMAX_SELECTED, o.SOFTMAX_ALL, o.SIGMOID, o.SIGMOID_NORMALISED]


def test_top_k_by_hand():
    s = np.array([[0.0, 2.0, 2.0, -1.0], [np.nan, -np.inf, 3.0, -5.0], [-0.0, 0.0, -0.0, 0.0]])
    assert o.top_k(s, 3).tolist() == [[1, 2, 0], [2, 3, 0], [0, 1, 2]]


def test_gates_by_hand():
    s = np.log(np.array([[1.0, 2.0, 5.0, 8.0]]))
    ids = np.array([[3, 1]])
    assert np.allclose(o.gates(s, ids, o.SOFTMAX_SELECTED), [[0.8, 0.2]])
    assert np.allclose(o.gates(s, ids, o.SOFTMAX_ALL), [[0.5, 0.125]])
    assert np.allclose(o.gates(s, ids, o.SIGMOID), [[8 / 9, 2 / 3]])
    assert np.allclose(o.gates(s, ids, o.SIGMOID_NORMALISED), [[4 / 7, 3 / 7]])
    assert (o.gates(np.full((1, 4), -np.inf), ids, o.SOFTMAX_SELECTED) == 0).all()
    assert (o.gates(s, ids, o.SIGMOID, mask=[0]) == 0).all()


def test_balance_of_even_routing_is_alpha():
    # every expert is picked equally often and every probability is 1/E, so E * sum (1/E)(1/E) = 1
    s, ids = np.zeros((8, 4)), np.arange(16).reshape(8, 2) % 4
    counts, prob, coef, loss = o.balance(s, ids, o.SOFTMAX_ALL, 0.5)
    assert counts.tolist() == [[4, 4, 4, 4]] and np.allclose(prob, 0.25) and np.isclose(loss, 0.5)
    assert np.allclose(coef, 0.5 * 4 * 0.25 / 8)
    _, _, _, both = o.balance(s, ids, o.SOFTMAX_ALL, 0.5, offsets=[0, 4, 4, 8])
    assert np.isclose(both, 1.0)       # two sequences and an empty one


@pytest.mark.parametrize("gating", GATINGS)
def test_balance_gradient_is_the_differences(gating):
    rng = np.random.default_rng(gating)
    s = rng.normal(size=(7, 5)) * 2
    ids = o.top_k(s, 2)
    off, mask = [1, 3, 3, 6], [1, 1, 1, 0, 1, 1, 1]
    coef = o.balance(s, ids, gating, 0.3, off, mask)[2]
    ds = o.route_bwd(s, gating, coef=coef, offsets=off, mask=mask)
    h = 1e-6
    for t in range(7):
        for e in range(5):
            up, down = s.copy(), s.copy()
            up[t, e] += h
            down[t, e] -= h
            diff = (o.balance(up, ids, gating, 0.3, off, mask)[3] - o.balance(down, ids, gating, 0.3, off, mask)[3]) / (2 * h)
            assert abs(diff - ds[t, e]) < 1e-8


@pytest.mark.parametrize("gating", GATINGS)
def test_gate_gradient_is_the_differences(gating):
    rng = np.random.default_rng(10 + gating)
    s = rng.normal(size=(4, 6)) * 2
    ids = o.top_k(s, 3)
    a = rng.normal(size=(4, 3))
    dlog = a * o.gates(s, ids, gating)       # L = sum a g
    ds = o.route_bwd(s, gating, ids, dlog)
    h = 1e-6
    for t in range(4):
        for e in range(6):
            up, down = s.copy(), s.copy()
            up[t, e] += h
            down[t, e] -= h
            diff = ((o.gates(up, ids, gating) - o.gates(down, ids, gating)) * a).sum() / (2 * h)
            assert abs(diff - ds[t, e]) < 1e-8


def test_adamw_by_hand():
    # first step: m/(1-b1) = g, v/(1-b2) = g^2, so the step is lr * sign(g)
    w, m, v = o.adamw(np.array([1.0, -2.0]), np.array([4.0, -3.0]), np.zeros(2), np.zeros(2), 0.1, 0.9, 0.99, 1e-30, 0.5, 1)
    assert np.allclose(w, [1 - 0.05 - 0.1, -2 + 0.1 + 0.1])
    assert np.allclose(m, [0.4, -0.3]) and np.allclose(v, [0.16, 0.09])


def test_e4m3_numbers():
    assert o.E4M3[0] == 0 and o.E4M3[1] == 2.0 ** -9 and o.E4M3[8] == 2.0 ** -6 and o.E4M3[126] == 448 and np.isnan(o.E4M3[127])
    assert (np.diff(o.E4M3[:127]) > 0).all() and (o.E4M3[128:255] == -o.E4M3[:127]).all()


def test_shared_exponents_and_neighbours():
    x = np.zeros(70)
    x[3], x[40], x[65] = 448.0, 448.1, 1.0
    e = o.shared_exponents(x)
    assert e.tolist() == [127, 128, 127 - 8]
    low, high = o.neighbours(np.array([1.0, 1.05, 500.0]), np.array([127]))
    assert low.tolist() == [1.0, 1.0, 448.0] and high.tolist() == [1.0, 1.125, 448.0]
    assert o.shared_exponents(np.array([1.0, np.nan]))[0] == 255 and o.shared_exponents(np.array([np.inf]))[0] == 255


def test_noise_is_even_and_changes_with_the_seed():
    """Bits of places and of seeds look like coin tosses: each of 32 bits over 2^16 places is set half the time (6 sigma), and two seeds
    agree in half of their bits."""
    p = np.arange(1 << 16, dtype=np.uint64)
    a, b = o.noise(p, 1), o.noise(p, 2)
    n = len(p)
    for h in (a, a ^ b, a[1:] ^ a[:-1]):
        for bit in range(32):
            share = ((h >> np.uint64(bit)) & np.uint64(1)).mean()
            assert abs(share - 0.5) < 6 * 0.5 / np.sqrt(n), bit
    assert abs(np.corrcoef((a >> np.uint64(12)).astype(float), (a & np.uint64(0xfff)).astype(float))[0, 1]) < 6 / np.sqrt(n)
