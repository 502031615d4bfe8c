"""Activations and their slopes at infinities, NaN and the largest numbers of each type, through every kind of kernel."""
import pytest
import torch

from test_gpu_linear import ACTS, F64, TYPES, act64, b  # noqa: F401

pytestmark = pytest.mark.gpu


def ends(dtype):
    top = torch.finfo(dtype).max
    return torch.tensor([float("inf"), float("-inf"), float("nan"), top, -top, 1e4, -1e4, 100.0, -100.0, 0.0, -0.0], dtype=dtype, device="cuda")


def same(got, want, dtype):
    """Equal where the value is 0 or not finite, NaN for NaN; else to the tolerance of a function and its rounding."""
    got, want = got.double(), want.to(dtype).double()
    assert torch.equal(got.isnan(), want.isnan())
    keep = ~want.isnan()
    got, want = got[keep], want[keep]
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[want.isinf()], want[want.isinf()])
    keep = want.isfinite()
    # (binary32's sigma and Phi are 0 below 2^-126, and a number of 2^14 by them with it: 2^-112)
    assert ((got[keep] - want[keep]).abs() <= (2.0 ** -19 + torch.finfo(dtype).eps) * want[keep].abs() + 2.0 ** -100).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [1, 3, 40, 300, 5000])
def test_activations_at_the_ends(b, act, dtype, n):
    """z = bias (x is 0) at both infinities, NaN and the largest numbers.  -inf by GELU, its tanh form and SiLU is -inf times 0: NaN, as in the formula."""
    z = ends(dtype).repeat(n // 4 + 1)                   # (11 columns and up)
    m = len(z)
    for k in (8, 72):
        out, keep = b.linear_forward(torch.zeros(n, k, dtype=dtype, device="cuda"), torch.ones(m, k, dtype=dtype, device="cuda"), bias=z, activation=act, want_preact=True)
        same(keep, z.expand(n, m), dtype)
        same(out, act64(z.to(F64), act).expand(n, m), dtype)


LIMITS = {"relu": (1, 0), "sigmoid": (0, 0), "gelu": (1, 0), "gelu_tanh": (1, 0), "silu": (1, 0)}      # slopes far above and far below


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("n", [1, 40, 300])
def test_slopes_at_the_ends(b, act, dtype, n):
    """Far out the slope is its limit, at the infinities too (a z past the type's range is kept as one): one such z leaves the sums of its column finite."""
    row = ends(dtype)[:9].repeat(4)
    m = len(row)
    above, below = LIMITS[act]
    want = torch.where(row.isnan(), row.to(F64), torch.where(row > 0, above, below).to(F64)).expand(n, m)
    z, one = row.expand(n, m), torch.ones(n, m, dtype=dtype, device="cuda")
    gx, gw, gb = b.linear_backward(one, torch.ones(n, 16, dtype=dtype, device="cuda"), torch.eye(m, dtype=dtype, device="cuda")[:, :m][:, :16].contiguous(), preact=z, activation=act)
    same(gb, want.sum(0), dtype)
    same(gw, want.sum(0)[:, None].expand(m, 16), dtype)
    if not want[:, :9].isnan().all():
        # gx by the unit vectors: NaN columns make every sum NaN; without them the first 16 slopes are it
        good = ~row.isnan()
        gx, _, _ = b.linear_backward(one[:, good], torch.ones(n, 16, dtype=dtype, device="cuda"), torch.eye(int(good.sum()), 16, dtype=dtype, device="cuda"), preact=z[:, good], activation=act)
        same(gx, want[:, good][:, :16], dtype)


@pytest.mark.parametrize("n,m", [(3, 100), (20, 1000), (200, 300)])
@pytest.mark.parametrize("power", [-100, -111, -118, -124])
def test_small_binary32_operands(b, n, m, power):
    """Three parts of 8 bits hold what lies above 2^-134 (half the smallest bfloat16) of an operand: the usual bound and that much of every x more."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    k = 500
    x, w = torch.randn(n, k, generator=gen, device="cuda") * 2.0 ** power, torch.randn(m, k, generator=gen, device="cuda") * 2.0 ** 100
    want, s = x.to(F64) @ w.to(F64).t(), x.to(F64).abs() @ w.to(F64).abs().t()
    got = b.linear_forward(x, w).to(F64)
    assert ((got - want).abs() <= (k + 16) * 2.0 ** -24 * s + 2.0 ** -134 * w.to(F64).abs().sum(1)).all()
    _, gw, _ = b.linear_backward(w.t(), x.t(), x.new_empty(m, n), want_x=False, want_bias=False)
    assert ((gw.to(F64) - want.t()).abs() <= (k + 16) * 2.0 ** -24 * s.t() + 2.0 ** -134 * w.to(F64).abs().sum(1)[:, None]).all()
