"""AdamW at the edges of its numbers: the smallest eps, gradients that are not finite."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
b = pytest.importorskip("paper_2603_06626_amd.binding")

DEV = "cuda:0"


def tensors(n, bits, grad, kind="fp32"):
    z = lambda m, dtype: torch.zeros(m, dtype=dtype, device=DEV)  # noqa: E731
    state = torch.float32 if bits == 32 else torch.uint8
    kw = {} if bits == 32 else dict(m_exp=[z(-(-n // 32), torch.uint8)], v_exp=[z(-(-n // 32), torch.uint8)])
    param = torch.ones(n, device=DEV).to(torch.float32 if kind == "fp32" else torch.bfloat16)
    if kind == "master":
        kw["master"] = [param.float()]
    return b.AdamWTensors([param], [grad], [z(n, state)], [z(n, state)], **kw), param


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", ["fp32", "master", "bf16"])
def test_weights_without_moments_stay_under_the_smallest_eps(kind, bits):
    """m = v = 0 and no gradient: the step is 0 / eps = 0."""
    t, p = tensors(100, bits, torch.zeros(100, device=DEV), kind)
    for step in (1, 2, 1000):
        b.grouter_adamw(t, b.grouter_adamw_hyper(1e-3, 0.9, 0.99, float(np.finfo(np.float32).tiny), 0.0, step, seed=step))
    assert (p == 1).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_gradient_that_is_not_finite_spoils_its_weight_alone(bad, bits):
    grad = torch.full((100,), 1e-3, device=DEV)
    grad[40] = bad
    t, p = tensors(100, bits, grad)
    b.grouter_adamw(t, b.grouter_adamw_hyper(1e-3, 0.9, 0.99, 1e-8, 0.0, 1))
    q = p.cpu().numpy()
    # m is bad, its root infinite or NaN: inf * 0 or NaN
    assert np.isnan(q[40]) and (np.abs(np.delete(q, 40) - (1 - 1e-3)) < 1e-6).all()
