"""Scores to ids and gates, the balance loss, the gates' gradient and the way back to the scores, against the 64-bit oracle.

Tolerances.  An exponential of x costs |x| 2^-24 (the product with log2 e) and 2^-23 (the hardware's), its sum and the division as much
again: with |x| <= 40 at most 1e-5 of the value.  bf16 and fp16 outputs add half a step of their type.
"""
import numpy as np
import pytest

from oracle import router as o

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
b = pytest.importorskip("paper_2603_06626_amd.binding")

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
FP = 1e-5
GATINGS = [b.GATE_SOFTMAX_SELECTED, b.GATE_SOFTMAX_ALL, b.GATE_SIGMOID, b.GATE_SIGMOID_NORMALISED]


def make_scores(T, E, dtype, seed, wide=0, spread=2.0):
    """Scores on the GPU (in rows of a wider matrix of NaN where `wide`) and what they hold in 64 bits."""
    rng = np.random.default_rng(seed)
    s = torch.full((T, E + wide), float("nan"), dtype=dtype, device=DEV)
    s[:, :E] = torch.from_numpy(rng.normal(size=(T, E)) * spread).to(DEV).to(dtype)
    return s[:, :E], s[:, :E].double().cpu().numpy()


def close(got, ref, tol):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    bad = ~(np.abs(got - ref) <= tol) & ~np.isnan(ref)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], ref[bad][:5])


def route(s, k, gating, ids=torch.int32, mask=None):
    T = s.shape[0]
    i = torch.full((T, k), 77, dtype=ids, device=DEV)
    g = torch.full((T, k), float("nan"), dtype=torch.bfloat16, device=DEV)
    b.grouter_route(s, k, gating, i, g, token_mask=mask)
    return i, g


def check_route(s, ref, k, gating, ids=torch.int32, mask=None):
    i, g = route(s, k, gating, ids, None if mask is None else torch.from_numpy(mask).to(DEV))
    want = o.top_k(ref, k)
    assert np.array_equal(i.cpu().numpy().astype(np.int64), want)
    gates = o.gates(ref, want, gating, mask)
    close(g, gates, np.nan_to_num(np.abs(gates)) * (2.0 ** -8 + FP) + 1e-38)


# every number of lanes per token, full and ragged, with vector and single loads
SIZES = [(1, 1, 1), (3, 2, 2), (70, 7, 3), (67, 8, 8), (300, 8, 2), (33, 9, 4), (5, 16, 1), (40, 17, 5), (19, 33, 6), (67, 60, 5), (30, 64, 6), (18, 65, 7),
         (35, 128, 8), (9, 129, 4), (9, 256, 8), (5, 257, 3), (5, 300, 70), (5, 512, 8), (3, 513, 9), (3, 1000, 8), (2, 1024, 5),
         # both sides of the lines between forms: lists of 4, 8 and 16, rounds
         (33, 16, 16), (20, 64, 9), (20, 64, 16), (20, 64, 17), (9, 256, 12), (5, 300, 12), (5, 300, 13), (5, 512, 16), (3, 1024, 16), (3, 1024, 17)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("T,E,k", SIZES)
def test_route_sizes(T, E, k, dtype):
    for n, gating in enumerate(GATINGS):
        s, ref = make_scores(T, E, dtype, 100 * E + n, wide=(0, 8, 3, 0)[n])
        check_route(s, ref, k, gating, torch.uint8 if E <= 256 and n % 2 else torch.int32)


@pytest.mark.parametrize("E,k", [(8, 8), (24, 24), (128, 128), (1024, 1024)])
def test_route_takes_all_experts(E, k):
    s, ref = make_scores(6, E, torch.float32, E)
    check_route(s, ref, k, b.GATE_SOFTMAX_SELECTED)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("E", [8, 60, 128, 300, 1024])
def test_route_ties_go_to_the_lowest_index(E, dtype):
    rng = np.random.default_rng(E)
    v = rng.integers(-2, 3, size=(40, E)).astype(np.float64)
    v[0] = 0.0
    v[1] = -0.0
    v[2, ::2] = -0.0
    v[2, 1::2] = 0.0
    s = torch.from_numpy(v).to(DEV).to(dtype)
    assert (s[1].view(torch.int32 if dtype == torch.float32 else torch.int16) != 0).all()     # the minus is there
    check_route(s, v, min(7, E), b.GATE_SIGMOID)


@pytest.mark.parametrize("gating", GATINGS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_route_masks_infinities_and_nan(dtype, gating):
    E, k, inf, nan, low = 60, 4, np.inf, np.nan, torch.finfo(dtype).min
    v = np.random.default_rng(1).normal(size=(12, E))
    v[0] = -inf                         # nothing left
    v[1, 3:] = -inf                     # fewer than k left
    v[2] = low                          # all at the type's lowest value: even
    v[3, :-1] = low
    v[4] = nan
    v[5, 10] = nan                      # a NaN that is not picked
    v[6, :57] = nan                     # fewer than k numbers
    v[7, 20] = inf
    v[8, [5, 30]] = inf
    v[9, 2:] = nan
    v[9, :2] = -inf
    v[10] = -200.0 if dtype != torch.float16 else -200.0      # sigmoids that underflow
    v[10, 7] = -199.0
    v[11] = 300.0
    s = torch.from_numpy(v).to(DEV).to(dtype)
    ref = s.double().cpu().numpy()
    i, g = route(s, k, gating)
    want = o.top_k(ref, k)
    assert np.array_equal(i.cpu().numpy(), want)
    with np.errstate(all="ignore"):
        gates = o.gates(ref, want, gating)
    if gating in (b.GATE_SOFTMAX_SELECTED, b.GATE_SOFTMAX_ALL):
        gates[7] = gates[8] = nan       # inf - inf
        if gating == b.GATE_SOFTMAX_ALL:
            gates[[4, 5, 6, 9]] = nan
        else:
            gates[[4, 6, 9]] = nan      # a NaN is among the selected
    elif gating == b.GATE_SIGMOID_NORMALISED:
        gates[[4, 6, 9]] = nan
    got = g.double().cpu().numpy()
    rows = [0, 1, 2, 3, 10, 11] if gating != b.GATE_SIGMOID else [0, 1, 2, 3, 5, 7, 8, 10, 11]
    tol = np.abs(gates) * (2.0 ** -8 + FP) + 1e-38
    if gating == b.GATE_SIGMOID:
        tol[10] = np.abs(gates[10]) * (2.0 ** -8 + 200 * 2.0 ** -24 * 4)      # e^-200 is below fp32's range: 0
        tol[10] = np.maximum(tol[10], 1e-38)
    assert (np.abs(got - gates)[rows] <= tol[rows]).all(), (got[rows], gates[rows])
    if gating != b.GATE_SIGMOID:
        assert np.array_equal(np.isnan(got), np.isnan(gates))
    else:
        assert np.isnan(got[4]).all() and not np.isnan(got[5]).any() and np.isnan(got[6, 3]) and np.isnan(got[9, 2:]).all()


@pytest.mark.parametrize("gating", GATINGS)
def test_route_padding_tokens(gating):
    s, ref = make_scores(50, 24, torch.float32, 8)
    mask = (np.arange(50) % 3 > 0).astype(np.uint8)
    s[::3] = float("nan")
    ref[::3] = np.nan
    i, g = route(s, 4, gating, torch.uint8, torch.from_numpy(mask).to(DEV))
    assert (g[::3] == 0).all() and not torch.isnan(g).any()
    assert (i[::3].cpu().numpy() == np.arange(4)).all()
    check_route(s, ref, 4, gating, mask=mask)
    j, h = route(s, 4, gating, torch.uint8, torch.from_numpy(mask).to(DEV).bool())
    assert torch.equal(i, j) and torch.equal(g, h)


def test_route_offsets_past_32_bits():
    ld, T, E, k = 1 << 20, 4200, 64, 6
    wide = torch.empty((T, ld), dtype=torch.bfloat16, device=DEV)      # 8.8 GB, 4.4e9 elements
    s = wide[:, 4096:4096 + E]
    s.copy_(torch.randn((T, E), device=DEV))
    rows = [0, 2047, 2048, 4095, 4096, T - 1]
    i, g = route(s, k, b.GATE_SOFTMAX_SELECTED)
    ref = s.double().cpu().numpy()
    assert np.array_equal(i.cpu().numpy()[rows], o.top_k(ref[rows], k))
    ds = wide[:, :E]
    b.grouter_route_bwd(s.float().contiguous(), b.GATE_SOFTMAX_SELECTED, ds, topk_idx=i, dlog_gate=torch.ones((T, k), device=DEV))
    want = o.route_bwd(ref[rows], b.GATE_SOFTMAX_SELECTED, i.cpu().numpy()[rows], np.ones((len(rows), k)))
    close(ds[rows], want, np.abs(want) * 2.0 ** -8 + 2 * k * FP)


# ---- balance loss and gradients -----------------------------------------------------------------------------------


def balance(s, ids, gating, alpha, off=None, mask=None):
    T, E = s.shape
    S = 1 if off is None else len(off) - 1
    off = None if off is None else torch.tensor(off, dtype=torch.int64, device=DEV)
    out = dict(counts=torch.full((S, E), -7, dtype=torch.int32, device=DEV), **{n: torch.full((S, E), float("nan"), device=DEV) for n in ("prob", "coef")},
               loss=torch.full((1,), float("nan"), device=DEV))
    ws = torch.full((b.grouter_balance_bytes(T, E, S),), 255, dtype=torch.uint8, device=DEV)
    b.grouter_balance(s, gating, ids, alpha, out["counts"], out["prob"], out["coef"], out["loss"], ws, token_mask=mask, seq_offsets=off)
    return out, off


def check_balance(s, ref, ids, gating, off=None, mask=None, grad=torch.float32, with_gates=False):
    T, E = ref.shape
    k = ids.shape[1]
    ids_d = torch.from_numpy(ids).to(DEV)
    mask_d = None if mask is None else torch.from_numpy(mask).to(DEV)
    out, off_d = balance(s, ids_d, gating, 0.37, off, mask_d)
    counts, prob, coef, loss = o.balance(ref, ids.astype(np.int64), gating, 0.37, off, mask)
    assert np.array_equal(out["counts"].cpu().numpy(), counts)
    close(out["prob"], prob, FP * prob + 1e-30)
    close(out["coef"], coef, 4 * 2.0 ** -24 * coef)
    assert abs(out["loss"].item() - loss) <= FP * loss
    q = np.random.default_rng(T).normal(size=(T, k)).astype(np.float32) if with_gates else None
    ds = torch.full((T, E + 5), 9.0, dtype=grad, device=DEV)
    b.grouter_route_bwd(s, gating, ds[:, :E], topk_idx=ids_d if with_gates else None, dlog_gate=None if q is None else torch.from_numpy(q).to(DEV),
                        token_mask=mask_d, seq_offsets=off_d, coef=out["coef"])
    assert (ds[:, E:] == 9.0).all()      # what lies between the rows is left
    dense = o.route_bwd(ref, gating, coef=coef, offsets=off, mask=mask)
    full = dense if q is None else dense + o.route_bwd(ref, gating, ids.astype(np.int64), q.astype(np.float64), mask=mask)
    p = np.stack([o.probabilities(r, gating) if np.isfinite(r).all() else np.zeros(E) for r in ref])
    big = coef.max() if coef.size else 0.0
    tol = 4 * FP * p * big + np.abs(full) * HALF_STEP[grad] + (2.0 ** -25 if grad == torch.float16 else 0.0)
    if q is not None:
        tol = tol + 2 * FP * np.abs(q).sum(1, keepdims=True)
    close(ds[:, :E], full, tol)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("T,E,k", SIZES)
def test_balance_sizes(T, E, k, dtype):
    for n, gating in enumerate(GATINGS):
        s, ref = make_scores(T, E, dtype, 7 * E + n, wide=(0, 8, 3, 0)[n])
        ids = o.top_k(ref, k).astype(np.uint8 if E <= 256 and n % 2 else np.int32)
        check_balance(s, ref, ids, gating, grad=TYPES[n % 3], with_gates=n > 1)


@pytest.mark.parametrize("off", [[0, 90], [0, 0, 30, 30, 31, 90, 90], [5, 17, 60, 80], [90, 90], [0, 0], [44, 44, 45], list(range(91)),
                                 [0] * 200 + [50] * 100 + [90] * 3], ids=lambda v: str(len(v)))
@pytest.mark.parametrize("gating", [b.GATE_SOFTMAX_ALL, b.GATE_SIGMOID])
def test_balance_sequences(off, gating):
    s, ref = make_scores(90, 40, torch.float32, 5)
    ids = o.top_k(ref, 3).astype(np.int32)
    check_balance(s, ref, ids, gating, off)
    mask = (np.random.default_rng(2).random(90) < 0.6).astype(np.uint8)
    mask[30:45] = 0                       # whole sequences of padding
    s[torch.from_numpy(mask).to(DEV) == 0] = float("nan")
    ref[mask == 0] = np.nan
    check_balance(s, ref, ids, gating, off, mask, with_gates=True)


@pytest.mark.parametrize("E,k", [(5, 2), (8, 2), (16, 3), (60, 5), (128, 8), (300, 4), (1000, 3)])
@pytest.mark.parametrize("n", [3, 40, 300])
def test_balance_sequences_within_and_across_tiles(E, k, n):
    """Random cuts, cuts at multiples of 8 (where tiles of tokens end), empty sequences, padding."""
    T = 700
    rng = np.random.default_rng(E + n)
    off = np.sort(np.concatenate([rng.integers(0, T + 1, n), 8 * rng.integers(0, T // 8, n // 2), [128, 256, 512]]))
    s, ref = make_scores(T, E, torch.bfloat16, n)
    ids = np.argsort(-ref, axis=1, kind="stable")[:, :k].astype(np.int32)
    mask = (rng.random(T) < 0.8).astype(np.uint8)
    check_balance(s, ref, ids, b.GATE_SOFTMAX_ALL if n == 40 else b.GATE_SIGMOID_NORMALISED, off.tolist(), mask)


def test_balance_sequences_over_many_chunks():
    """Sequences of 1 to 20000 tokens over the whole grid of chunks, against 64-bit sums of torch."""
    T, E, k = 70001, 64, 6
    s = torch.randn((T, E), device=DEV) * 2 + torch.randn(E, device=DEV)
    ids = s.topk(k, dim=1).indices.int()
    off = [0, 1, 2, 500, 500, 20500, 20501, 20629, 40000, 60000, 70000]
    out, _ = balance(s, ids, b.GATE_SOFTMAX_SELECTED, 1.0, off)
    again, _ = balance(s, ids, b.GATE_SOFTMAX_SELECTED, 1.0, off)
    assert all(torch.equal(out[n], again[n]) for n in out)
    p, loss = torch.softmax(s.double(), 1), 0.0
    for i, (a, z) in enumerate(zip(off, off[1:])):
        c = torch.bincount(ids[a:z].reshape(-1).long(), minlength=E)
        assert torch.equal(out["counts"][i].long(), c)
        if z > a:
            mean = p[a:z].mean(0)
            assert ((out["prob"][i] - mean).abs() <= FP * mean).all()
            loss += E * float((c.double() / (k * (z - a)) * mean).sum())
        else:
            assert (out["prob"][i] == 0).all() and (out["coef"][i] == 0).all()
    assert abs(out["loss"].item() - loss) <= FP * loss


def test_balance_ids_outside_and_repeated():
    s, ref = make_scores(30, 20, torch.float32, 3)
    ids = np.random.default_rng(4).integers(-3, 25, size=(30, 4)).astype(np.int32)
    ids[:, 1] = ids[:, 0]
    ids[7] = -1                            # a token whose ids are all bad
    ids[8] = 3                             # and one whose ids are all the same
    for gating in GATINGS:
        check_balance(s, ref, ids, gating, with_gates=True)


@pytest.mark.parametrize("gating", GATINGS)
def test_gradient_of_closed_experts_is_zero(gating):
    s, ref = make_scores(20, 30, torch.float32, 6)
    shut = np.random.default_rng(7).random((20, 30)) < 0.4
    shut[0] = True
    ref[shut] = -np.inf
    s = torch.from_numpy(ref).float().to(DEV)
    ids = o.top_k(ref, 3).astype(np.int32)
    out, _ = balance(s, torch.from_numpy(ids).to(DEV), gating, 1.0)
    ds = torch.empty((20, 30), device=DEV)
    b.grouter_route_bwd(s, gating, ds, coef=out["coef"])
    assert not torch.isnan(ds).any() and (ds.cpu().numpy()[shut] == 0).all()
    b.grouter_route_bwd(s, gating, ds, topk_idx=torch.from_numpy(ids).to(DEV), dlog_gate=torch.ones((20, 3), device=DEV))
    assert not torch.isnan(ds).any()


def test_gradient_into_columns_of_the_same_matrix():
    wide = torch.randn((300, 150), device=DEV)
    s, ds = wide[:, 10:70], wide[:, 70:130]
    keep = wide.clone()
    out, _ = balance(s, s.topk(3, dim=1).indices.int(), b.GATE_SIGMOID, 1.0)
    b.grouter_route_bwd(s, b.GATE_SIGMOID, ds, coef=out["coef"])
    alone = torch.empty((300, 60), device=DEV)
    b.grouter_route_bwd(keep[:, 10:70], b.GATE_SIGMOID, alone, coef=out["coef"])
    assert torch.equal(ds, alone) and torch.equal(wide[:, :70], keep[:, :70]) and torch.equal(wide[:, 130:], keep[:, 130:])
    with pytest.raises(b.GrouterError):
        b.grouter_route_bwd(s, b.GATE_SIGMOID, wide[:, 69:129], coef=out["coef"])


@pytest.mark.parametrize("gating", GATINGS)
def test_gradient_is_the_differences_of_the_gates(gating):
    """L = sum a g over the gates in 64 bits, by differences of the oracle's gates; the kernel gets a g as the gradient by their logs."""
    s, ref = make_scores(12, 16, torch.float32, 21)
    ids = o.top_k(ref, 4)
    a = np.random.default_rng(3).normal(size=(12, 4))
    q = a * o.gates(ref, ids, gating)
    ds = torch.empty((12, 16), device=DEV)
    b.grouter_route_bwd(s, gating, ds, topk_idx=torch.from_numpy(ids.astype(np.int32)).to(DEV), dlog_gate=torch.from_numpy(q).float().to(DEV))
    got, h = ds.double().cpu().numpy(), 1e-5
    for t in range(12):
        for e in range(16):
            up, down = ref.copy(), ref.copy()
            up[t, e] += h
            down[t, e] -= h
            diff = ((o.gates(up, ids, gating) - o.gates(down, ids, gating)) * a)[t].sum() / (2 * h)
            assert abs(diff - got[t, e]) <= 2 * FP * np.abs(q[t]).sum() + 1e-8


@pytest.mark.parametrize("gating", [b.GATE_SOFTMAX_SELECTED, b.GATE_SIGMOID_NORMALISED])
@pytest.mark.parametrize("E", [8, 60, 256])
def test_gradient_of_the_only_selected_expert_is_zero(gating, E):
    """Its gate is 1 whatever its score."""
    s, ref = make_scores(500, E, torch.float32, E)
    ids = torch.from_numpy(o.top_k(ref, 1).astype(np.int32)).to(DEV)
    ds = torch.ones((500, E), device=DEV)
    b.grouter_route_bwd(s, gating, ds, topk_idx=ids, dlog_gate=torch.randn((500, 1), device=DEV))
    assert (ds == 0).all()


# ---- gradient by the gates ----------------------------------------------------------------------------------------


@pytest.mark.parametrize("T,E,k,d", [(1, 1, 1, 8), (1, 8, 2, 16), (7, 5, 5, 72), (33, 60, 5, 1032), (64, 8, 1, 512), (20, 64, 6, 2048), (5, 128, 8, 8200), (300, 16, 3, 24),
                                     (3, 200, 100, 264)])
def test_gate_gradient(T, E, k, d):
    rng = np.random.default_rng(d)
    ids = torch.from_numpy(rng.integers(0, E, size=(T, k)).astype(np.int32)).to(DEV)
    plan = torch.empty(b.grouter_plan_bytes(T, k, E), dtype=torch.uint8, device=DEV)
    b.grouter_plan_build(ids, E, plan)
    dY, rows = (torch.from_numpy(rng.normal(size=(n, d))).to(DEV).bfloat16() for n in (T, T * k))
    out = torch.full((T, k), float("nan"), device=DEV)
    b.grouter_gate_bwd(plan, T, k, E, dY, rows, out)
    s2r = b.grouter_plan_views(plan, T, k, E)[3].cpu().numpy()
    a, r = dY.double().cpu().numpy(), rows.double().cpu().numpy()
    ref = o.gate_bwd(a, r, s2r, k)
    bound = o.gate_bwd(np.abs(a), np.abs(r), s2r, k)         # a sum of d products, each rounded at most d/64 + 8 times
    close(out, ref, (d / 8 + 16) * 2.0 ** -24 * bound)


def test_gate_gradient_with_another_plan_writes_nothing():
    T, E, k, d = 10, 8, 2, 64
    plan = torch.zeros(b.grouter_plan_bytes(T, k, E) + 4096, dtype=torch.uint8, device=DEV)
    b.grouter_plan_build(torch.zeros((T, k), dtype=torch.int32, device=DEV), E, plan)
    out = torch.full((T, k + 1), 5.0, device=DEV)
    b.grouter_gate_bwd(plan, T, k + 1, E, torch.zeros((T, d), dtype=torch.bfloat16, device=DEV),
                       torch.zeros((T * (k + 1), d), dtype=torch.bfloat16, device=DEV), out)
    assert (out == 5.0).all()
