"""The router, the balance loss and AdamW where numbers get large: tokens, sequences, elements past 2^31 and places past 2^32; graphs that
replay side by side; the phases that the timing API keeps for them.  References are torch's in 64 bits, tolerances those of the small
tests (1e-5 for exponentials and their shares)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
b = pytest.importorskip("paper_2603_06626_amd.binding")

DEV, FP = "cuda:0", 1e-5


def balance_buffers(T, E, S):
    new = lambda dtype=torch.float32: torch.empty((S, E), dtype=dtype, device=DEV)  # noqa: E731
    return dict(counts=new(torch.int32), prob=new(), coef=new(), loss=torch.empty(1, device=DEV),
                ws=torch.empty(b.grouter_balance_bytes(T, E, S), dtype=torch.uint8, device=DEV))


def test_millions_of_tokens_in_many_sequences():
    T, E, k, S = 1_000_003, 64, 6, 30000
    s = torch.randn((T, E), device=DEV)
    ids, g = torch.empty((T, k), dtype=torch.uint8, device=DEV), torch.empty((T, k), dtype=torch.bfloat16, device=DEV)
    b.grouter_route(s, k, b.GATE_SOFTMAX_SELECTED, ids, g)
    v, i = s.sort(dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), i[:, :k])
    ref = torch.softmax(v[:, :k].double(), 1)
    assert ((g.double() - ref).abs() <= ref * (2.0 ** -8 + FP)).all()
    off = torch.arange(S + 1, device=DEV) * 33
    off[-1] = T
    out = balance_buffers(T, E, S)
    b.grouter_balance(s, b.GATE_SOFTMAX_SELECTED, ids, 1.0 / S, **out, seq_offsets=off)
    p = torch.softmax(s.double(), 1)
    run = torch.cat([torch.zeros((1, E), device=DEV, dtype=torch.float64), p.cumsum(0)])
    n = (off[1:] - off[:-1]).double()[:, None]
    prob = (run[off[1:]] - run[off[:-1]]) / n
    assert ((out["prob"] - prob).abs() <= FP * prob + 1e-9).all()      # (differences of running sums of up to 1e6 / 64: 2^-53 of 2e4)
    hot = torch.zeros((T, E), dtype=torch.int64, device=DEV).scatter_add_(1, ids.long(), torch.ones((T, k), dtype=torch.int64, device=DEV))
    run = torch.cat([torch.zeros((1, E), device=DEV, dtype=torch.int64), hot.cumsum(0)])
    counts = run[off[1:]] - run[off[:-1]]
    assert torch.equal(out["counts"].long(), counts)
    loss = (E / S * (counts.double() / (k * n) * prob).sum()).item()
    assert abs(out["loss"].item() - loss) <= FP * loss
    ds = torch.empty((T, E), device=DEV)
    b.grouter_route_bwd(s, b.GATE_SOFTMAX_SELECTED, ds, seq_offsets=off, coef=out["coef"])
    c = out["coef"].double()[torch.searchsorted(off, torch.arange(T, device=DEV), right=True) - 1]
    want = p * (c - (c * p).sum(1, keepdim=True))
    assert ((ds - want).abs() <= 4 * FP * p * c.amax(1, keepdim=True)).all()


def test_adamw_past_32_bits():
    """Three tensors of 2^31 + 77 elements: gradients of 0.5 move weights of 1 by 1e-3, which bf16 takes one way or the other."""
    n = (1 << 31) + 77
    new = lambda dtype, fill, m=n: torch.full((m,), fill, dtype=dtype, device=DEV)  # noqa: E731
    param, grad = [new(torch.bfloat16, 1.0) for _ in range(3)], [new(torch.bfloat16, 0.5) for _ in range(3)]
    m, v = ([new(torch.uint8, 0) for _ in range(3)] for _ in range(2))
    exps = [[new(torch.uint8, 0, -(-n // 32)) for _ in range(3)] for _ in range(2)]
    t = b.AdamWTensors(param, grad, m, v, m_exp=exps[0], v_exp=exps[1])
    b.grouter_adamw(t, b.grouter_adamw_hyper(1e-3, 0.9, 0.99, 1e-8, 0.0, 1, seed=3))
    part = 1 << 24
    for x in param:
        for a in (0, n // 2, n - part):
            y = x[a:a + part].float()
            assert set(y.unique().tolist()) == {1.0, 1.0 - 2.0 ** -8}
            # the mean of 2^24 draws of 0 or 2^-8 with probability 0.256: standard error 2^-8 * 0.44 / 2^12 = 4e-7
            assert abs(y.double().mean().item() - 0.999) < 6 * 4.2e-7
    assert not torch.equal(param[0][:part], param[1][:part]) and not torch.equal(param[0][:part], param[2][:part])
    assert all((x[-77:] > 0).all() and (x[:77] > 0).all() for x in v)


def test_graphs_side_by_side():
    """Two captured losses with workspaces of their own, replayed on two streams at once."""
    kept = []
    for T in (5000, 5777):
        E, k, S = 96, 6, 9
        s = torch.randn((T, E), device=DEV)
        ids, off = s.topk(k, 1).indices.int(), torch.linspace(0, T, S + 1, device=DEV).long()
        out, ds = balance_buffers(T, E, S), torch.empty((T, E), device=DEV)

        def both(s=s, ids=ids, off=off, out=out, ds=ds):
            b.grouter_balance(s, b.GATE_SIGMOID, ids, 0.1, **out, seq_offsets=off)
            b.grouter_route_bwd(s, b.GATE_SIGMOID, ds, seq_offsets=off, coef=out["coef"])

        both()
        torch.cuda.synchronize()
        results = [out[n] for n in ("counts", "prob", "coef", "loss")] + [ds]
        ref = [x.clone() for x in results]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both()
        kept.append((graph, results, ref, torch.cuda.Stream(), both))
    for _ in range(5):
        for graph, results, _, stream, _ in kept:
            for x in results:
                x.zero_()
        torch.cuda.synchronize()
        for graph, _, _, stream, _ in kept:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, results, ref, _, _ in kept:
            assert all(torch.equal(x, y) for x, y in zip(results, ref))


def test_phases_are_timed():
    T, E, k, d = 64, 16, 2, 64
    s, x = torch.randn((T, E), device=DEV), torch.zeros((T, d), dtype=torch.bfloat16, device=DEV)
    ids, g = torch.empty((T, k), dtype=torch.int32, device=DEV), torch.empty((T, k), dtype=torch.bfloat16, device=DEV)
    plan, dlog = torch.empty(b.grouter_plan_bytes(T, k, E), dtype=torch.uint8, device=DEV), torch.empty((T, k), device=DEV)
    w = [torch.zeros(64, device=DEV) for _ in range(4)]
    out, ds = balance_buffers(T, E, 1), torch.empty((T, E), device=DEV)
    b.grouter_timing_enable(True)
    b.grouter_timing_read()
    b.grouter_route(s, k, 0, ids, g)
    b.grouter_plan_build(ids, E, plan)
    b.grouter_balance(s, 0, ids, 1.0, **out)
    b.grouter_gate_bwd(plan, T, k, E, x, torch.zeros((T * k, d), dtype=torch.bfloat16, device=DEV), dlog)
    b.grouter_route_bwd(s, 0, ds, topk_idx=ids, dlog_gate=dlog, coef=out["coef"])
    b.grouter_adamw(b.AdamWTensors(w[:1], w[1:2], w[2:3], w[3:]), b.grouter_adamw_hyper(1e-3, 0.9, 0.99, 1e-8, 0.0, 1))
    times = b.grouter_timing_read()
    b.grouter_timing_enable(False)
    assert all(times[p][1] == 1 and times[p][0] > 0 for p in ("route", "balance", "gate_bwd", "route_bwd", "adamw"))


def test_grids_past_32_bits_of_threads():
    """More threads than one dimension of a grid takes: 2^26 + 3 tokens of 520 equal scores, 2^26 + 24 slots of 8 values."""
    T, E, k = (1 << 26) + 3, 520, 2
    s = torch.zeros((T, E), dtype=torch.bfloat16, device=DEV)
    s[-1, 7] = s[1 << 25, 519] = s[0, 300] = 1.0
    ids, g = torch.full((T, k), -1, dtype=torch.int32, device=DEV), torch.zeros((T, k), dtype=torch.bfloat16, device=DEV)
    b.grouter_route(s, k, b.GATE_SIGMOID_NORMALISED, ids, g)
    want = torch.arange(k, device=DEV).expand(T, k).clone().int()
    for t, e in ((0, 300), (1 << 25, 519), (T - 1, 7)):
        want[t] = torch.tensor([e, 0])
    assert torch.equal(ids, want)
    assert (g[1:1 << 25] == 0.5).all() and (g[-1].float().sum() - 1).abs() < 2.0 ** -7
    del g, want
    ds = torch.full((T, E), 5.0, dtype=torch.bfloat16, device=DEV)
    b.grouter_route_bwd(s, b.GATE_SIGMOID, ds, topk_idx=ids, dlog_gate=torch.ones((T, k), device=DEV))
    assert (ds[1:1 << 25, :2] == 0.5).all() and (ds[1:1 << 25, 2:8] == 0).all() and (ds[-1, 1:7] == 0).all() and ds[-1, 0] == 0.5 and ds[-1, 7] < 0.5
    del s, ds, ids
    torch.cuda.empty_cache()
    T, E, k, d = (1 << 23) + 3, 16, 8, 8
    plan = torch.empty(b.grouter_plan_bytes(T, k, E), dtype=torch.uint8, device=DEV)
    b.grouter_plan_build((torch.arange(T * k, device=DEV).view(T, k) % E).int(), E, plan)
    rows = (torch.arange(T * k, device=DEV) % 251).to(torch.bfloat16)[:, None].expand(-1, d).contiguous()
    dlog = torch.empty((T, k), device=DEV)
    b.grouter_gate_bwd(plan, T, k, E, torch.ones((T, d), dtype=torch.bfloat16, device=DEV), rows, dlog)
    at = b.grouter_plan_views(plan, T, k, E)[3].long()
    assert torch.equal(dlog.view(-1), (8 * (at % 251)).float())
