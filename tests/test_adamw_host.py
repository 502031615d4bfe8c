"""strads_adamw_step and strads_adamw_unpack: what they refuse, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding, build
    build.build()
    binding.load()
    return binding


def _config(b, **kw):
    c = b.AdamWConfig(param_type=0, grad_type=0, state_bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, l1=0.0,
                      grad_scale=1.0, step=1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _tensors(b, tensors=2, **kw):
    list_ = (b.AdamWTensor * tensors)()
    for i in range(tensors):
        t = list_[i]
        t.param, t.grad, t.m, t.v, t.n = 0x100000 + i * 0x10000, 0x200000, 0x300000, 0x400000, 1000      # never dereferenced
        t.m_scale, t.v_scale = 0x500000, 0x600000
    for k, v in kw.items():
        setattr(list_[tensors - 1], k, v)
    return list_


INVALID = [dict(state_bits=16), dict(param_type=3), dict(param_type=-1), dict(grad_type=1), dict(param_type=1, grad_type=2), dict(lr=-1.0),
           dict(lr=float("nan")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0),
           dict(eps=1e-60), dict(weight_decay=-1.0), dict(l1=-1.0), dict(l1=float("inf")), dict(grad_scale=float("nan")), dict(step=0)]


@pytest.mark.parametrize("kw", INVALID, ids=str)
def test_bad_configurations_are_refused(b, kw):
    assert b.load().strads_adamw_step(C.byref(_config(b, **kw)), _tensors(b), 2) == -1


BAD_TENSORS = [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=-1), dict(param=0x100002), dict(grad=0x200002),
               dict(m=0x300001), dict(master=0x700000), dict(param=0x100000), dict(param=0x100000 + 4 * 999)]


@pytest.mark.parametrize("kw", BAD_TENSORS, ids=str)
def test_bad_tensors_are_refused(b, kw):
    """NULL and misaligned arrays, a master beside 32-bit parameters, the same parameters twice or in part."""
    assert b.load().strads_adamw_step(C.byref(_config(b)), _tensors(b, **kw), 2) == -1


def test_other_refusals(b):
    lib = b.load()
    assert lib.strads_adamw_step(None, _tensors(b), 2) == -1
    assert lib.strads_adamw_step(C.byref(_config(b)), None, 2) == -1
    assert lib.strads_adamw_step(C.byref(_config(b)), _tensors(b), -1) == -1
    assert lib.strads_adamw_step(C.byref(_config(b)), _tensors(b), 0) == 0
    assert lib.strads_adamw_step(C.byref(_config(b)), (b.AdamWTensor * 3)(), 3) == 0    # nothing there
    big = _tensors(b)
    big[1].n = (1 << 40) + 1
    assert lib.strads_adamw_step(C.byref(_config(b)), big, 2) == -7
    for kw in (dict(m_scale=None), dict(v_scale=None), dict(m_scale=0x500002)):
        assert lib.strads_adamw_step(C.byref(_config(b, state_bits=8)), _tensors(b, **kw), 2) == -1
    # masters for one of two
    assert lib.strads_adamw_step(C.byref(_config(b, param_type=1, grad_type=1)), _tensors(b, master=0x700000), 2) == -1
    # an unsorted list with an overlap in the middle
    t = _tensors(b, 3)
    t[0].param, t[1].param, t[2].param = 0x150000, 0x110000, 0x110000 + 3996
    assert lib.strads_adamw_step(C.byref(_config(b)), t, 3) == -1
    outs = (C.c_void_p * 2)(0x700000, 0x710000)
    assert lib.strads_adamw_unpack(None, outs, outs, 2, None) == -1
    assert lib.strads_adamw_unpack(_tensors(b), None, outs, 2, None) == -1
    assert lib.strads_adamw_unpack(_tensors(b, m_scale=None), outs, outs, 2, None) == -1
    assert lib.strads_adamw_unpack(_tensors(b), (C.c_void_p * 2)(0x700000, None), outs, 2, None) == -1
    assert lib.strads_adamw_unpack(_tensors(b), (C.c_void_p * 2)(0x700002, 0x710000), outs, 2, None) == -1
    assert lib.strads_adamw_unpack(_tensors(b), outs, outs, 0, None) == 0


def test_the_class_refuses_what_it_cannot_take(b):
    import torch
    p = torch.zeros(10)
    with pytest.raises(ValueError):
        b.AdamW([p])                                     # not on a CUDA device
    with pytest.raises(ValueError):
        b.AdamW([])
    with pytest.raises(ValueError):
        b.AdamW([p], bits=16)
    with pytest.raises(TypeError):
        b.AdamW([p.double()])
    with pytest.raises(ValueError):
        b.AdamW([p], masters=[p])
