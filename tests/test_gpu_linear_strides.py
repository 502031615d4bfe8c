"""Results of linear layers that lie two elements apart in rows of an odd length."""
import pytest
import torch

from test_gpu_linear import TYPES, b, matrix  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,m", [(3, 50, 3), (40, 90, 33), (150, 200, 131), (2305, 64, 2311)])
def test_results_two_elements_apart_in_odd_rows(b, n, k, m, dtype):
    """Every second column of a buffer with an odd width, and every second row of one with an odd height by columns: no two results at one place."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, w, g = matrix(n, k, dtype, gen), matrix(m, k, dtype, gen, scale=k ** -0.5), matrix(n, m, dtype, gen)
    want, z = b.linear_forward(x, w, activation="gelu", want_preact=True)
    grads = b.linear_backward(g, x, w, preact=z, activation="gelu")
    new = lambda r, c: torch.full((r, 2 * c - 1), 77.0, dtype=dtype, device="cuda")
    turned = lambda r, c: torch.full((c, 2 * r - 1), 77.0, dtype=dtype, device="cuda")
    for make, take in ((new, lambda t: t[:, ::2]), (turned, lambda t: t[:, ::2].t())):
        out, keep, gx, gw = make(n, m), make(n, m), make(n, k), make(m, k)
        b.linear_forward(x, w, activation="gelu", out=take(out), preact=take(keep))
        b.linear_backward(g, x, w, preact=z, activation="gelu", grad_x=take(gx), grad_w=take(gw))
        for got, v in ((out, want), (keep, z), (gx, grads[0]), (gw, grads[1])):
            tol = 2.0 ** -10 if dtype == torch.float32 else 4 * torch.finfo(dtype).eps      # (other tiles: other orders of the sums)
            assert ((take(got).double() - v.double()).abs() <= tol * (1 + v.double().abs().amax())).all()
            take(got).fill_(77.0)
            assert (got == 77.0).all()
