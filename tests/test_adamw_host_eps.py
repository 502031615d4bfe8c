"""strads_adamw_step: the smallest eps, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("eps", [1e-39, 1e-40, 1e-45, 1.17e-38])
def test_an_eps_whose_inverse_is_no_number_is_refused(b, eps):
    """Where both moments are 0 the step is 0 / eps: with an inverse of infinity it would be NaN.  (The list is bad too, so that nothing is ever launched.)"""
    c = b.AdamWConfig(param_type=0, grad_type=0, state_bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=eps, grad_scale=1.0, step=1)
    huge = b.AdamWTensor(param=0x100000, grad=0x200000, m=0x300000, v=0x400000, n=(1 << 40) + 1)      # -7 where the configuration is taken
    assert b.load().strads_adamw_step(C.byref(c), C.byref(huge), 1) == -1
    for taken in (2.0 ** -126, 1e-37, 1e-8, 1.0):
        c.eps = taken
        assert b.load().strads_adamw_step(C.byref(c), C.byref(huge), 1) == -7
