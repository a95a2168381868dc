"""The optimizer's numbers are refused where the fp32 numbers that the step computes with would not be theirs."""
import numpy as np
import pytest

from paper_2603_06626_amd import binding as b

GOOD = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1)
TINY = float(np.finfo(np.float32).tiny)


@pytest.fixture(scope="module", autouse=True)
def library():
    import os

    if not os.path.exists(b.LIB_PATH):
        from paper_2603_06626_amd.build import build_library

        build_library()


@pytest.mark.parametrize("bad", [dict(eps=1e-50), dict(eps=1e-45), dict(eps=1e-39), dict(eps=TINY * (1 - 1e-6)), dict(eps=1e39), dict(eps=-1e-8), dict(eps=float("nan")),
                                 dict(lr=1e39), dict(lr=1e38, beta1=0.99), dict(lr=-1e39), dict(lr=1e30, weight_decay=1e30), dict(lr=1e300, weight_decay=1e300),
                                 dict(lr=0.0, weight_decay=float("inf")), dict(grad_scale=1e39), dict(grad_scale=-1e39), dict(beta1=1 - 1e-9), dict(beta2=1 - 1e-9)], ids=str)
def test_numbers_that_fp32_does_not_hold(bad):
    with pytest.raises(b.GrouterError) as e:
        b.grouter_adamw_hyper(**{**GOOD, **bad})
    assert e.value.code == b.ERR_INVALID_ARG


@pytest.mark.parametrize("good", [dict(eps=TINY), dict(eps=1e-37), dict(eps=1e30), dict(lr=0.0), dict(lr=1e-60), dict(lr=1e37), dict(grad_scale=0.0), dict(grad_scale=-1.0),
                                  dict(beta1=0.0, beta2=0.0), dict(beta2=1 - 1e-7), dict(step=1 << 40)], ids=str)
def test_numbers_at_the_edge(good):
    h = b.grouter_adamw_hyper(**{**GOOD, **good})
    assert all(np.isfinite(getattr(h, n)) for n, _ in h._fields_[:9]) and h.eps >= np.float32(TINY) and h.beta2 < 1


def test_refused_numbers_leave_the_structure():
    h = b.grouter_adamw_hyper(**GOOD)
    import ctypes

    before = bytes(h)
    assert b.lib().grouter_adamw_hyper_set(1e-3, 0.9, 0.99, 1e-50, 0.1, 1, 1.0, 7, ctypes.byref(h)) == b.ERR_INVALID_ARG
    assert bytes(h) == before
