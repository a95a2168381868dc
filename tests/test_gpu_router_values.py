"""The balance loss and the gradient by the scores where scores are far from 0: experts closed by the type's lowest value or by a large
negative number, alone, all of a row, and beside ordinary tokens of the same sequence.

Tolerances.  The difference to the row's largest is rounded once (2^-24 of it) and its product with log2 e once more; the hardware's exponential
costs 2^-23, sum and division as much again.  What is within 40 of the largest is off by at most 1e-5 of its value, what is further is
below 1e-17.  The gradient p (c - <c, p>) has p twice: 4e-5 of p times the largest coefficient.
"""
import numpy as np
import pytest

from oracle import router as o

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
b = pytest.importorskip("paper_2603_06626_amd.binding")

DEV, FP, ALPHA, K = "cuda:0", 1e-5, 0.37, 3
TYPES = [torch.float32, torch.bfloat16, torch.float16]
GATINGS = [b.GATE_SOFTMAX_SELECTED, b.GATE_SOFTMAX_ALL, b.GATE_SIGMOID, b.GATE_SIGMOID_NORMALISED]


def make_rows(E, dtype, seed):
    """Scores [T, E] as a tensor and in 64 bits: every second token is an ordinary one."""
    rng = np.random.default_rng(seed)
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    special = []
    for far in (low, -1e9, -1e10, -1e12, -1e30, high, 1e10, 2e38):
        if abs(far) > high:
            continue
        special.append(np.full(E, far))                                      # nothing but it: even
        some = rng.normal(size=E)
        some[rng.random(E) < 0.6] = far
        some[1] = far
        special.append(some)                                                 # closed to some, or far above the others
        one = np.full(E, far)
        one[E // 2] = 1.5
        special.append(one)
        special.append(np.where(np.arange(E) % 2 > 0, far, -np.inf))         # beside -inf
        if far < 0:
            special.append(np.where(np.arange(E) % 3 > 0, far, low))
    rows = np.empty((2 * len(special), E))
    rows[0::2] = rng.normal(size=(len(special), E)) * 2
    rows[1::2] = special
    scores = torch.from_numpy(rows).to(dtype)
    return scores.to(DEV), scores.double().numpy()


def close(got, want, tol, what):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("gating", GATINGS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("E", [5, 8, 60, 128, 300, 1024])
def test_scores_far_from_zero(E, dtype, gating):
    s, ref = make_rows(E, dtype, E)
    T = len(ref)
    p = np.stack([o.probabilities(r, gating) for r in ref])
    assert np.isfinite(p).all() and (p.sum(1) > 0.999).all()
    ids = o.top_k(ref, K)
    ids_d = torch.from_numpy(ids.astype(np.int32)).to(DEV)
    q = np.random.default_rng(3).normal(size=(T, K)).astype(np.float32)
    for off in (None, [0, T], [0, 1, 2, 5, 9, T - 2], list(range(0, T + 1, 2))):
        S = 1 if off is None else len(off) - 1
        off_d = None if off is None else torch.tensor(off, dtype=torch.int64, device=DEV)
        counts = torch.empty((S, E), dtype=torch.int32, device=DEV)
        prob, coef, loss = torch.empty((S, E), device=DEV), torch.empty((S, E), device=DEV), torch.empty(1, device=DEV)
        ws = torch.empty(b.grouter_balance_bytes(T, E, S), dtype=torch.uint8, device=DEV)
        b.grouter_balance(s, gating, ids_d, ALPHA, counts, prob, coef, loss, ws, seq_offsets=off_d)
        rc, rp, rf, rl = o.balance(ref, ids, gating, ALPHA, off)
        assert np.array_equal(counts.cpu().numpy(), rc)
        close(prob, rp, FP * rp + 1e-17, "prob")
        close(coef, rf, 4 * 2.0 ** -24 * rf, "coef")
        assert abs(loss.item() - rl) <= FP * rl
        ds = torch.full((T, E), float("nan"), device=DEV)
        b.grouter_route_bwd(s, gating, ds, seq_offsets=off_d, coef=coef)
        close(ds, o.route_bwd(ref, gating, coef=rf, offsets=off), (4 * FP * p + 1e-17) * rf.max(), "balance gradient")
    ds = torch.full((T, E), float("nan"), device=DEV)
    b.grouter_route_bwd(s, gating, ds, topk_idx=ids_d, dlog_gate=torch.from_numpy(q).to(DEV))
    with np.errstate(over="ignore"):
        want = o.route_bwd(ref, gating, ids, q.astype(np.float64))
    close(ds, want, 2 * FP * np.abs(q).sum(1, keepdims=True), "gate gradient")
