"""Gradients through an activation whose gz = gout act'(z) or scale lies where 16-bit types end."""
import pytest
import torch

from test_gpu_linear import ACTS, F64, TYPES, b, close, half_step, matrix, slope64  # noqa: F401

pytestmark = pytest.mark.gpu


def check_gradient(b, gout, x, w, z, act, scale, lost, slope_error=2.0 ** -20, relative=0.0):
    """As check_backward of test_gpu_linear.py, with scale a factor of the sums.  lost(|gz|, dim): what an element of gz may lose beside eps / 2 of itself, where a
    sum goes along dim.  slope_error: of the slope, as a part of the largest; relative: as a part of itself."""
    gx, gw, gb = b.linear_backward(gout, x, w, preact=z, activation=act, scale=scale)
    t = x.dtype
    u = 0.0 if t == torch.float32 else torch.finfo(t).eps / 2
    g, s = gout.to(F64), abs(scale)
    gz = g * slope64(z.to(F64), act)
    own = gz.abs() * (2.0 ** -22 + relative) + slope_error * g.abs()
    e = own + u * gz.abs()
    (n, k), m = x.shape, w.shape[0]
    for got, want, mag, err, terms in ((gx, gz @ w.to(F64), gz.abs() @ w.to(F64).abs(), (e + lost(gz.abs(), 1)) @ w.to(F64).abs(), m),
                                       (gw, gz.t() @ x.to(F64), gz.abs().t() @ x.to(F64).abs(), (e + lost(gz.abs(), 0)).t() @ x.to(F64).abs(), n),
                                       (gb, gz.sum(0), gz.abs().sum(0), own.sum(0), n)):
        want, tol = scale * want, s * ((terms + 16) * 2.0 ** -24 * mag + err)
        tol = tol + half_step(want.abs() + tol, t)
        beyond = want.abs() - tol > torch.finfo(t).max * (1 + torch.finfo(t).eps / 4)      # a result that its type does not hold is an infinity
        assert torch.equal(got[beyond].double(), want[beyond].sign() * float("inf"))
        near = (want.abs() + tol > torch.finfo(t).max) & ~beyond
        close(got[~beyond & ~near], want[~beyond & ~near], tol[~beyond & ~near])


# few rows, few columns, one tile, several, and pairs of CTAs
SHAPES = [(3, 40, 64), (64, 40, 3), (100, 64, 72), (150, 301, 77), (2340, 200, 2568)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("size,scale", [(100.0, 1024.0), (1000.0, 100.0), (1e-3, 2.0 ** -10), (3e-3, 1.0 / 8192), (1.0, 1e-4)])
def test_scale_is_outside_of_the_rounding(b, act, size, scale, dtype):
    """gout of `size` by a scale that leaves binary16's range before the products, with results inside it.  gz may lose half a subnormal's step, 2^-25."""
    for n, k, m in SHAPES[:4] if act != "silu" else SHAPES:
        gen = torch.Generator(device="cuda").manual_seed(n)
        gout, z = matrix(n, m, dtype, gen, scale=size), matrix(n, m, dtype, gen)
        other = min(100.0, 100.0 / (size * scale) / max(m, n) ** 0.5)
        x, w = matrix(n, k, dtype, gen, scale=other), matrix(m, k, dtype, gen, "cols", scale=other)
        check_gradient(b, gout, x, w, z, act, scale, lambda gz, dim: 2.0 ** -25 if dtype == torch.float16 else 0.0)
