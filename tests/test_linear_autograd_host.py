"""Layers record nothing for autograd: tensors that would need it are refused (no GPU needed)."""
import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding, build
    build.build()
    binding.load()
    return binding


def test_forward_refuses_what_requires_a_gradient(b):
    new = lambda *s: torch.zeros(*s)
    for which in ("x", "w", "bias", "residual"):
        args = dict(x=new(4, 8), w=new(3, 8), bias=new(3), residual=new(4, 3))
        args[which].requires_grad_(True)
        with pytest.raises(RuntimeError, match="autograd"):
            b.linear_forward(**args)
        for relaxed in (torch.no_grad, torch.inference_mode):
            with relaxed(), pytest.raises(ValueError):   # goes on, to the check of the device
                b.linear_forward(**args)


def test_backward_refuses_what_requires_a_gradient(b):
    new = lambda *s: torch.zeros(*s)
    for which in ("grad_out", "x", "w", "preact"):
        args = dict(grad_out=new(4, 3), x=new(4, 8), w=new(3, 8), preact=new(4, 3))
        args[which].requires_grad_(True)
        with pytest.raises(RuntimeError, match="autograd"):
            b.linear_backward(**args)
        with torch.no_grad(), pytest.raises(ValueError):
            b.linear_backward(**args)
