"""One training step around the expert layer, run as a program would: scores, ids and gates, plan, layer forward and backward, the gates'
gradient, the balance loss, the gradient by the scores, AdamW over the router's and the experts' weights.  The gradients are checked
against autograd of the same step in 64 bits on the CPU, a captured step against the eager one."""
import numpy as np
import pytest

from oracle import router as o

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
b = pytest.importorskip("paper_2603_06626_amd.binding")

DEV, BF = "cuda:0", torch.bfloat16
GATINGS = [b.GATE_SOFTMAX_SELECTED, b.GATE_SOFTMAX_ALL, b.GATE_SIGMOID, b.GATE_SIGMOID_NORMALISED]
OFFSETS, ALPHA = [0, 40, 41, 90], 0.05


class Step:
    """Buffers of one step on one batch; run() enqueues it whole."""

    def __init__(self, gating, T=96, d=64, f=128, E=8, k=2, states=32, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.gating, self.T, self.d, self.f, self.E, self.k = gating, T, d, f, E, k
        rnd = lambda *s, sigma: torch.randn(s, generator=g, device=DEV) * sigma  # noqa: E731
        new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device=DEV)  # noqa: E731
        self.x, self.dY = rnd(T, d, sigma=1.0).to(BF), rnd(T, d, sigma=1.0).to(BF)
        self.Ws = rnd(d, E, sigma=d ** -0.5)
        self.W = [rnd(E, d, f, sigma=d ** -0.5), rnd(E, d, f, sigma=d ** -0.5), rnd(E, f, d, sigma=f ** -0.5)]     # master copies
        self.Wb = [w.to(BF) for w in self.W]
        self.dW = [torch.empty_like(w) for w in self.Wb]
        self.dWs = torch.empty_like(self.Ws)
        self.scores, self.dscores = new(T, E), new(T, E)
        self.ids, self.gates, self.dlog = new(T, k, dtype=torch.int32), new(T, k, dtype=BF), new(T, k)
        self.y, self.dX = new(T, d, dtype=BF), new(T, d, dtype=BF)
        self.off = torch.tensor(OFFSETS, device=DEV)
        S = len(OFFSETS) - 1
        self.counts, self.prob, self.coef, self.loss = new(S, E, dtype=torch.int32), new(S, E), new(S, E), new(1)
        ws = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)  # noqa: E731
        self.plan, self.ctx = ws(b.grouter_plan_bytes(T, k, E)), ws(b.grouter_ctx_bytes(T, k, d, f))
        self.scratch, self.bws = ws(b.grouter_bwd_scratch_bytes(T, k, d, f)), ws(b.grouter_balance_bytes(T, E, S))
        zeros = lambda t: torch.zeros_like(t, dtype=torch.float32 if states == 32 else torch.uint8)  # noqa: E731
        exps = lambda ts: None if states == 32 else [ws(-(-t.numel() // 32)).zero_() for t in ts]  # noqa: E731
        self.experts = b.AdamWTensors(self.Wb, self.dW, [zeros(w) for w in self.W], [zeros(w) for w in self.W], master=self.W, m_exp=exps(self.W),
                                      v_exp=exps(self.W))
        self.router = b.AdamWTensors([self.Ws], [self.dWs], [zeros(self.Ws)], [zeros(self.Ws)], m_exp=exps([self.Ws]), v_exp=exps([self.Ws]))
        self.hyper = torch.zeros(48, dtype=torch.uint8, device=DEV)

    def run(self, update=True):
        torch.matmul(self.x.float(), self.Ws, out=self.scores)
        b.grouter_route(self.scores, self.k, self.gating, self.ids, self.gates)
        b.grouter_plan_build(self.ids, self.E, self.plan)
        b.grouter_moe_fwd(self.plan, self.x, self.gates, *self.Wb, self.y, self.ctx)
        b.grouter_moe_bwd(self.plan, self.x, self.gates, *self.Wb, self.dY, self.ctx, self.dX, *self.dW, self.scratch)
        b.grouter_moe_gate_bwd(self.plan, self.E, self.f, self.dY, self.ctx, self.dlog)
        b.grouter_balance(self.scores, self.gating, self.ids, ALPHA, self.counts, self.prob, self.coef, self.loss, self.bws, seq_offsets=self.off)
        b.grouter_route_bwd(self.scores, self.gating, self.dscores, topk_idx=self.ids, dlog_gate=self.dlog, seq_offsets=self.off, coef=self.coef)
        torch.matmul(self.x.float().t(), self.dscores, out=self.dWs)
        if update:
            b.grouter_adamw(self.experts, self.hyper)
            b.grouter_adamw(self.router, self.hyper)

    def all(self):
        return [self.y, self.dX, *self.dW, self.dWs, self.loss, self.counts, self.Ws, *self.W, *self.Wb] + [t for x in (self.experts, self.router) for n in (2, 3)
                                                                                                         for t in x._held[n]]


@pytest.mark.parametrize("gating", GATINGS)
def test_gradients_are_those_of_the_whole_step(gating):
    s = Step(gating)
    s.run(update=False)
    x, dY, ids = s.x.double().cpu(), s.dY.double().cpu(), s.ids.long().cpu()
    Ws = s.Ws.double().cpu().requires_grad_()
    W1, W3, W2 = (w.double().cpu() for w in s.Wb)
    scores = x @ Ws
    assert np.array_equal(ids.numpy(), o.top_k(s.scores.double().cpu().numpy(), s.k))
    over = {b.GATE_SOFTMAX_SELECTED: lambda: torch.softmax(scores.gather(1, ids), 1), b.GATE_SOFTMAX_ALL: lambda: torch.softmax(scores, 1).gather(1, ids),
            b.GATE_SIGMOID: lambda: torch.sigmoid(scores.gather(1, ids)),
            b.GATE_SIGMOID_NORMALISED: lambda: torch.sigmoid(scores.gather(1, ids)) / torch.sigmoid(scores.gather(1, ids)).sum(1, keepdim=True)}
    r = over[gating]()
    outs = torch.stack([(torch.nn.functional.silu(x @ W1[e]) * (x @ W3[e])) @ W2[e] for e in range(s.E)], 1)      # [T, E, d]
    y = (r[:, :, None] * outs.gather(1, ids[:, :, None].expand(-1, -1, s.d))).sum(1)
    p = torch.softmax(scores, 1) if gating < 2 else torch.sigmoid(scores) / torch.sigmoid(scores).sum(1, keepdim=True)
    loss = 0.0
    for a, z in zip(OFFSETS, OFFSETS[1:]):
        share = torch.bincount(ids[a:z].reshape(-1), minlength=s.E).double() / (s.k * (z - a))
        loss = loss + ALPHA * s.E * (share * p[a:z].mean(0)).sum()
    ((y * dY).sum() + loss).backward()
    # the layer keeps its outputs in bf16 (half a step of 2^-8 each, and again in H and G, U before them): 1e-2 of the largest, as for the
    # layer's own gradients
    got, ref = s.dWs.double().cpu(), Ws.grad
    assert (got - ref).abs().max() <= 1e-2 * ref.abs().max()
    assert abs(s.loss.item() - float(loss.detach())) <= 1e-5 * float(loss.detach())
    assert (s.y.double().cpu() - y.detach()).abs().max() <= 1e-2 * y.detach().abs().max()


@pytest.mark.parametrize("states", [32, 8])
def test_captured_steps_equal_eager_ones(states):
    a, e = Step(b.GATE_SOFTMAX_SELECTED, states=states), Step(b.GATE_SOFTMAX_SELECTED, states=states)
    a.run(update=False)          # libraries load what they need before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for step in range(1, 5):
        h = b.grouter_adamw_hyper(1e-3, 0.9, 0.99, 1e-8, 0.1, step, seed=step)
        for s in (a, e):
            s.hyper.copy_(h.tensor())
            s.x.copy_(torch.randn(s.x.shape, generator=torch.Generator().manual_seed(step)))
        graph.replay()
        torch.cuda.synchronize()
        e.run()
        torch.cuda.synchronize()
        for i, (p, q) in enumerate(zip(a.all(), e.all())):
            assert torch.equal(p, q), (step, i)


def test_first_step_moves_every_weight_by_the_learning_rate():
    """Every weight moves by about the learning rate in the first step, against its gradient's sign."""
    s = Step(b.GATE_SIGMOID_NORMALISED)
    before = [w.clone() for w in s.W] + [s.Ws.clone()]
    s.hyper.copy_(b.grouter_adamw_hyper(1e-3, 0.9, 0.99, 1e-12, 0.0, 1, seed=1).tensor())
    s.run()
    for w, old, g in zip(s.W + [s.Ws], before, s.dW + [s.dWs]):
        moved = (w - old)[g.abs() > 1e-6]
        # lr sign(g), within the rounding of the weight (at most 4: 2^-22) and the step's own 1e-5
        assert ((moved + 1e-3 * torch.sign(g[g.abs() > 1e-6].float())).abs() <= 1e-8 * 1e3 * 1e-3 + 2.0 ** -22 + 1e-6).all()


def test_two_streams_at_once():
    """Independent steps on two streams, each with workspaces of its own, give what they give alone."""
    alone, pair, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(2):
        s = Step(GATINGS[i], seed=i)
        s.run(update=False)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in s.all()])
        pair.append(Step(GATINGS[i], seed=i))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, stream in zip(pair, streams):
            with torch.cuda.stream(stream):
                s.run(update=False)
    torch.cuda.synchronize()
    for s, ref in zip(pair, alone):
        assert all(torch.equal(p, q) for p, q in zip(s.all(), ref))
