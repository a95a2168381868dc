"""Which tensors the calls of the router, the loss, the gate gradient and the optimizer take, without a GPU: stand-ins for tensors on two
devices, and a stand-in for the library that records what gets through."""
import types

import pytest

from paper_2603_06626_amd import binding as b

torch = pytest.importorskip("torch")
F32, BF, I32, I64, U8 = torch.float32, torch.bfloat16, torch.int32, torch.int64, torch.uint8


class Fake:
    is_cuda = True
    addresses = iter(range(1 << 20, 1 << 40, 1 << 20))

    def __init__(self, shape, dtype, device=0):
        self.shape, self.dtype, self.index, self.at = torch.Size(shape), dtype, device, next(Fake.addresses)
        self.device = types.SimpleNamespace(index=device)

    def get_device(self):
        return self.index

    def data_ptr(self):
        return self.at

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize


class Cpu(Fake):
    is_cuda = False

    def __init__(self, like):
        super().__init__(like.shape, like.dtype, -1)


T, E, k, S, d, f = 6, 8, 2, 3, 16, 24


def tensors(name):
    """Arguments of a call as keywords: tensors and plain values."""
    rows = dict(scores=Fake((T, E), F32), topk_idx=Fake((T, k), I32), token_mask=Fake((T,), U8))
    if name == "grouter_route":
        return dict(rows, k=k, gating=0, gate_w=Fake((T, k), BF))
    per = dict(seq_offsets=Fake((S + 1,), I64), coef=Fake((S, E), F32))
    if name == "grouter_route_bwd":
        return dict(rows, gating=0, dscores=Fake((T, E), BF), dlog_gate=Fake((T, k), F32), **per)
    if name == "grouter_balance":
        return dict(rows, gating=0, alpha=0.1, counts=Fake((S, E), I32), prob=Fake((S, E), F32), loss=Fake((1,), F32), ws=Fake((1 << 16,), U8), **per)
    plan = dict(plan_ws=Fake((1 << 16,), U8), E=E, dY=Fake((T, d), BF), dlog_gate=Fake((T, k), F32))
    if name == "grouter_gate_bwd":
        return dict(plan, T=T, k=k, inp=Fake((T * k, d), BF))
    if name == "grouter_moe_gate_bwd":
        return dict(plan, f=f, ctx_ws=Fake((1 << 16,), U8))
    one = [[Fake((64,), F32)] for _ in range(4)]
    return dict(tensors=types.SimpleNamespace(count=1, _held=one, _array=None, kind=0, grad_dtype=0, bits=32), hyper=Fake((48,), U8), grad_scale=Fake((1,), F32))


CALLS = ["grouter_route", "grouter_route_bwd", "grouter_balance", "grouter_gate_bwd", "grouter_moe_gate_bwd", "grouter_adamw"]


@pytest.fixture
def calls(monkeypatch):
    seen = []
    library = types.SimpleNamespace(grouter_plan_bytes=lambda *a: 4096)
    for name in CALLS:
        setattr(library, name, lambda *a, name=name: seen.append((name, a)) or 0)
    monkeypatch.setattr(b, "_lib", library)
    monkeypatch.setattr(b, "_current", (lambda: 0, lambda device: 77 + device))
    return seen


@pytest.mark.parametrize("name", CALLS)
def test_tensors_on_one_device_get_through(calls, name):
    args = tensors(name)
    getattr(b, name)(**args)
    assert len(calls) == 1 and calls[0][0] == name and calls[0][1][-1] == 77
    for key, t in args.items():
        if isinstance(t, Fake):
            assert t.at in calls[0][1], key


@pytest.mark.parametrize("name,key", [(n, key) for n in CALLS for key, t in tensors(n).items() if isinstance(t, Fake)])
def test_a_tensor_on_another_device_is_refused(calls, name, key):
    for other in (lambda t: Fake(t.shape, t.dtype, 1), Cpu):
        args = tensors(name)
        args[key] = other(args[key])
        with pytest.raises(ValueError):
            getattr(b, name)(**args)
    assert not calls


@pytest.mark.parametrize("name", ["grouter_route", "grouter_balance"])
def test_all_on_another_device_than_the_current_one(calls, name):
    args = {key: Fake(t.shape, t.dtype, 1) if isinstance(t, Fake) else t for key, t in tensors(name).items()}
    with pytest.raises(ValueError):
        getattr(b, name)(**args)
    getattr(b, name)(**args, stream=types.SimpleNamespace(device=types.SimpleNamespace(index=1), cuda_stream=5))
    assert calls[0][1][-1] == 5 and len(calls) == 1


def test_gradients_of_gates_without_their_ids(calls):
    with pytest.raises(ValueError):
        b.grouter_route_bwd(Fake((T, E), F32), 0, Fake((T, E), F32), dlog_gate=Fake((T, k), F32))
    assert not calls
