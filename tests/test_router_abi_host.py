"""What the router's, the balance loss's, the gate gradient's and the optimizer's entry points refuse, all on the host: no call here gets
as far as a launch, so the addresses are never used."""
import ctypes

import pytest

from paper_2603_06626_amd import binding as b

FAKE = 1 << 20


@pytest.fixture(scope="module")
def L():
    import os

    if not os.path.exists(b.LIB_PATH):
        from paper_2603_06626_amd.build import build_library

        build_library()
    return b.lib()


ROUTE = dict(scores=FAKE, dtype=0, ld=64, T=4, E=64, k=2, gating=0, mask=None, ids=FAKE, idx=0, gates=FAKE, stream=None)
BAD_ROUTE = [dict(scores=None), dict(dtype=3), dict(dtype=-1), dict(ld=63), dict(T=0), dict(T=-1), dict(T=1 << 31), dict(E=0), dict(E=1025, ld=2000), dict(k=0),
             dict(k=65), dict(gating=4), dict(gating=-1), dict(ids=None), dict(idx=2), dict(idx=1, E=257, ld=257), dict(gates=None), dict(gates=FAKE + 1),
             dict(scores=FAKE + 2), dict(scores=FAKE + 1, dtype=1), dict(ids=FAKE + 2), dict(T=1 << 30, k=2), dict(ld=1 << 40)]


@pytest.mark.parametrize("bad", BAD_ROUTE, ids=str)
def test_route_refuses(L, bad):
    assert L.grouter_route(*{**ROUTE, **bad}.values()) == b.ERR_INVALID_ARG


BWD = dict(scores=FAKE, dtype=0, ld=64, T=4, E=64, gating=0, mask=None, ids=FAKE, idx=0, k=2, dlog=FAKE, off=None, S=1, coef=FAKE, ds=FAKE + 65536, ddt=0, dld=64,
           stream=None)
BAD_BWD = [dict(scores=None), dict(ds=None), dict(ddt=3), dict(dld=63), dict(dlog=None, coef=None), dict(ids=None), dict(k=0), dict(k=65), dict(idx=7), dict(S=0),
           dict(S=2), dict(S=(1 << 24) + 1, off=FAKE), dict(off=FAKE + 4), dict(coef=FAKE + 2), dict(gating=9), dict(ds=FAKE), dict(ds=FAKE + 4 * 64 * 4 - 4),
           dict(dlog=FAKE + 1), dict(E=1025, ld=1025, dld=1025), dict(T=0), dict(ds=FAKE + 65537, ddt=1)]


@pytest.mark.parametrize("bad", BAD_BWD, ids=str)
def test_route_bwd_refuses(L, bad):
    assert L.grouter_route_bwd(*{**BWD, **bad}.values()) == b.ERR_INVALID_ARG


BALANCE = dict(scores=FAKE, dtype=0, ld=64, T=4, E=64, k=2, gating=0, mask=None, ids=FAKE, idx=0, off=None, S=1, alpha=0.1, counts=FAKE, prob=FAKE, coef=FAKE,
               loss=FAKE, ws=FAKE, ws_bytes=1 << 20, stream=None)
BAD_BALANCE = [dict(scores=None), dict(dtype=5), dict(ld=1), dict(T=0), dict(E=1025, ld=1025), dict(k=0), dict(k=65), dict(gating=4), dict(ids=None), dict(idx=3),
               dict(S=0), dict(S=2), dict(off=FAKE + 4), dict(counts=None), dict(prob=None), dict(coef=None), dict(loss=None), dict(ws=None), dict(ws=FAKE + 64),
               dict(counts=FAKE + 1), dict(idx=1, E=300, ld=300)]


@pytest.mark.parametrize("bad", BAD_BALANCE, ids=str)
def test_balance_refuses(L, bad):
    assert L.grouter_balance(*{**BALANCE, **bad}.values()) == b.ERR_INVALID_ARG


def test_balance_workspace(L):
    need = b.grouter_balance_bytes(4, 64, 1)
    assert need > 0 and need % 256 == 0
    assert L.grouter_balance(*{**BALANCE, "ws_bytes": need - 1}.values()) == b.ERR_WORKSPACE_TOO_SMALL
    assert b.grouter_balance_bytes(0, 64, 1) == 0 and b.grouter_balance_bytes(4, 1025, 1) == 0 and b.grouter_balance_bytes(4, 64, 0) == 0
    assert b.grouter_balance_bytes(4, 64, (1 << 24) + 1) == 0 and b.grouter_balance_bytes(1 << 31, 64, 1) == 0
    assert b.grouter_balance_bytes(1 << 20, 256, 1000) > 1000 * 256 * 8


@pytest.mark.parametrize("bad", [dict(plan=None), dict(T=0), dict(k=9), dict(d=0), dict(d=12), dict(dY=None), dict(dY=FAKE + 8), dict(rows=None), dict(rows=FAKE + 2),
                                 dict(out=None), dict(out=FAKE + 2)], ids=str)
def test_gate_bwd_refuses(L, bad):
    good = dict(plan=FAKE, T=4, k=2, E=8, d=64, dY=FAKE, rows=FAKE, out=FAKE, stream=None)
    assert L.grouter_gate_bwd(*{**good, **bad}.values()) == b.ERR_INVALID_ARG


def test_moe_gate_bwd_refuses(L):
    need = b.grouter_ctx_bytes(4, 2, 64, 64)
    good = dict(plan=FAKE, T=4, k=2, E=8, d=64, f=64, dY=FAKE, ctx=FAKE, n=need, out=FAKE, stream=None)
    for bad in (dict(plan=None), dict(ctx=None), dict(ctx=FAKE + 16), dict(f=60), dict(d=60), dict(dY=None), dict(out=None), dict(k=9)):
        assert L.grouter_moe_gate_bwd(*{**good, **bad}.values()) == b.ERR_INVALID_ARG, bad
    assert L.grouter_moe_gate_bwd(*{**good, "n": need - 1}.values()) == b.ERR_WORKSPACE_TOO_SMALL


TENSOR = dict(param=FAKE, master=None, grad=FAKE, m=FAKE, v=FAKE, m_exp=None, v_exp=None, n=100)


def adamw(L, tensor=None, count=1, kind=0, grad=0, bits=32, hyper=True, dev=None, scale=None, list_=True):
    h = b.grouter_adamw_hyper(1e-3, 0.9, 0.99, 1e-8, 0.1, 1)
    t = (b._AdamWTensor * 1)(b._AdamWTensor(*{**TENSOR, **(tensor or {})}.values()))
    return L.grouter_adamw(t if list_ else None, count, kind, grad, bits, ctypes.byref(h) if hyper else None, dev, scale, None)


@pytest.mark.parametrize("bad", [dict(count=-1), dict(list_=False), dict(kind=3), dict(kind=-1), dict(grad=2), dict(bits=16), dict(hyper=False), dict(dev=FAKE),
                                 dict(hyper=False, dev=FAKE + 2), dict(scale=FAKE + 1), dict(kind=1), dict(tensor=dict(master=FAKE)), dict(bits=8),
                                 dict(bits=8, tensor=dict(m_exp=FAKE)), dict(tensor=dict(m_exp=FAKE)), dict(tensor=dict(v_exp=FAKE)), dict(tensor=dict(param=None)),
                                 dict(tensor=dict(grad=None)), dict(tensor=dict(m=None)), dict(tensor=dict(v=None)), dict(tensor=dict(n=-1)),
                                 dict(tensor=dict(n=1 << 41)), dict(tensor=dict(param=FAKE + 8)), dict(tensor=dict(grad=FAKE + 2)), dict(tensor=dict(m=FAKE + 4)),
                                 dict(tensor=dict(v=FAKE + 4)), dict(kind=1, tensor=dict(master=FAKE + 4))], ids=str)
def test_adamw_refuses(L, bad):
    assert adamw(L, **bad) == b.ERR_INVALID_ARG


def test_adamw_of_nothing(L):
    assert adamw(L, count=0, list_=False) == b.OK
    assert adamw(L, tensor=dict(n=0, param=None, grad=None, m=None, v=None)) == b.OK


@pytest.mark.parametrize("bad", [dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=float("inf")),
                                 dict(lr=float("nan")), dict(weight_decay=float("inf")), dict(grad_scale=float("nan"))], ids=str)
def test_hyper_refuses(L, bad):
    with pytest.raises(b.GrouterError):
        b.grouter_adamw_hyper(**{**dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1), **bad})


def test_hyper_numbers(L):
    h = b.grouter_adamw_hyper(2e-3, 0.9, 0.99, 1e-8, 0.1, 3, grad_scale=0.5, seed=-1)
    assert abs(h.step_size - 2e-3 / (1 - 0.9 ** 3)) < 1e-9 and abs(h.inv_root_correction - (1 - 0.99 ** 3) ** -0.5) < 1e-6
    assert abs(h.one_minus_beta2 - 0.01) < 1e-9 and abs(h.decay - 2e-4) < 1e-10 and h.grad_scale == 0.5 and h.seed == 0xffffffff
    assert ctypes.sizeof(b.AdamWHyper) == 48 and h.tensor().numel() == 48


def test_binding_refuses_cpu_tensors_and_shapes():
    import torch

    s, ids, g = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        b.grouter_route(s, 2, b.GATE_SIGMOID, ids, g)
    x = [torch.zeros(32)]
    with pytest.raises(ValueError):
        b.AdamWTensors(x, x, x, x)
    with pytest.raises(ValueError):
        b.AdamWTensors(x, x, x, [])


def test_phases_of_the_new_operators(L):
    assert b.PHASES[16:] == ("route", "route_bwd", "balance", "gate_bwd", "adamw")


@pytest.mark.parametrize("ds,dld,ok", [(FAKE + 64 * 4, 128, True), (FAKE + 64 * 4 - 4, 128, False), (FAKE + 64 * 4 + 4, 128, False), (FAKE + 10 * 512 + 256, 128, True),
                                       (FAKE - 256, 128, True), (FAKE - 252, 128, False), (FAKE + 64 * 4, 129, False), (FAKE + 3 * 512 + 256, 129, True)])
def test_columns_of_one_matrix_do_not_overlap(L, ds, dld, ok):
    """scores: four rows of 64 fp32 in rows of 128; refused calls return before the next check fails (S = 0), which both do."""
    case = {**BWD, "ld": 128, "ds": ds, "dld": dld}
    assert L.grouter_route_bwd(*{**case, "S": 0}.values()) == b.ERR_INVALID_ARG
    if not ok:
        assert L.grouter_route_bwd(*case.values()) == b.ERR_INVALID_ARG


def test_tensors_and_stream_have_to_be_on_one_device(monkeypatch):
    class On:
        def __init__(self, index):
            self.index = self.cuda_stream = index
            self.device = self

        def get_device(self):
            return self.index

    monkeypatch.setattr(b, "_current", (lambda: 0, lambda device: 77 + device))
    assert b._stream_for(On(0)) == 77 and b._stream_for(On(1), On(1)) == 1
    for t, stream in ((On(1), None), (On(0), On(1))):
        with pytest.raises(ValueError):
            b._stream_for(t, stream)
