"""Gradients through an activation whose gz = gout act'(z) or scale lies where 16-bit types end."""
import pytest
import torch

from test_gpu_linear import ACTS, F64, TYPES, b, close, half_step, matrix, slope64  # noqa: F401

pytestmark = pytest.mark.gpu


def check_gradient(b, gout, x, w, z, act, scale, lost, slope_error=2.0 ** -20, relative=0.0):
    """As check_backward of test_gpu_linear.py, with scale a factor of the sums.  lost(|gout|, dim): what an element of gz may lose beside eps / 2 of itself, where a
    sum goes along dim.  slope_error: of the slope, as a part of the largest; relative: as a part of itself."""
    gx, gw, gb = b.linear_backward(gout, x, w, preact=z, activation=act, scale=scale)
    t = x.dtype
    u = 0.0 if t == torch.float32 else torch.finfo(t).eps / 2
    g, s = gout.to(F64), abs(scale)
    gz = g * slope64(z.to(F64), act)
    own = gz.abs() * (2.0 ** -22 + relative) + slope_error * g.abs()
    e = own + u * gz.abs()
    (n, k), m = x.shape, w.shape[0]
    for got, want, mag, err, terms in ((gx, gz @ w.to(F64), gz.abs() @ w.to(F64).abs(), (e + lost(g.abs(), 1)) @ w.to(F64).abs(), m),
                                       (gw, gz.t() @ x.to(F64), gz.abs().t() @ x.to(F64).abs(), (e + lost(g.abs(), 0)).t() @ x.to(F64).abs(), n),
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
        check_gradient(b, gout, x, w, z, act, scale, lambda g, dim: 2.0 ** -25 if dtype == torch.float16 else 0.0)


def of_the_largest(g, dim):
    """A power of two of the sum's own line brings its largest |gout| to 2^14 .. 2^15, so half a subnormal's step of gz, 2^-25, is at most 2^-39 of it."""
    return 2.0 ** -39 * g.where(g.isfinite(), torch.zeros_like(g)).amax(dim, keepdim=True)


@pytest.mark.parametrize("shape", [(8192, 24, 40), (40, 24, 8192), (8192, 3, 4), (4, 3, 8192), (1, 300, 8192), (8192, 300, 1), (1000, 129, 1001)])
@pytest.mark.parametrize("outlier", [False, True])
def test_gradients_below_the_types_range(b, shape, outlier):
    """gout = 1e-4 by slopes of 1e-4, all of one sign: 1e-8, a third of what binary16 rounds to 0, adds up to what it does hold.  One row and one column of
    gout at the other end of the range: the others keep what they had."""
    n, k, m = shape
    gen = torch.Generator(device="cuda").manual_seed(n)
    gout = (1e-4 * (1 + torch.rand(n, m, generator=gen, device="cuda"))).half()
    if outlier:
        gout[n // 2] = 3e4
        gout[:, m // 2] = -2e4
    z = (-9.2 - 0.3 * torch.rand(n, m, generator=gen, device="cuda")).half()
    x, w = ((1 + torch.rand(*s, generator=gen, device="cuda")).half() for s in ((n, k), (m, k)))
    # exp(-|z|): the product with log2 e is off by 2^-24 of 14, its power of two by 2^-22, inverse and products by 2^-22: below 2^-18 of the slope
    check_gradient(b, gout, x, w, z, "sigmoid", 1.0, of_the_largest, slope_error=0.0, relative=2.0 ** -18)
    if not outlier and 8192 in (n, m):
        gx, gw, _ = b.linear_backward(gout, x, w, preact=z, activation="sigmoid")
        assert ((gx if m == 8192 else gw) > 0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_slopes_above_one_by_the_largest_numbers(b, act, dtype):
    """gout at the type's largest number by slopes up to 1.13, x and w small enough for results inside the range (bfloat16, whose range is that of the sums: 2^118)."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    n, k, m = 70, 40, 33
    top = 65504.0 if dtype == torch.float16 else 2.0 ** 118
    gout = torch.full((n, m), top, device="cuda").to(dtype)
    z = (1.5 + torch.rand(n, m, generator=gen, device="cuda")).to(dtype)
    x, w = matrix(n, k, dtype, gen, scale=0.01), matrix(m, k, dtype, gen, scale=0.01)
    check_gradient(b, gout, x, w, z, act, 2.0 ** -8, of_the_largest)


def test_rows_of_noughts_and_of_what_is_not_finite(b):
    """A row without a gradient gives noughts; an infinity or NaN stays in its row of gx and its column's row of gw."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, k, m = 130, 72, 90
    gout, z, x, w = (matrix(*s, torch.float16, gen) for s in ((n, m), (n, m), (n, k), (m, k)))
    gout[5] = 0
    gout[:, 7] = 0
    clean = b.linear_backward(gout, x, w, preact=z, activation="gelu")
    assert not clean[0][5].any() and not clean[1][7].any() and not clean[2][7].any()
    for value in (float("inf"), float("nan")):
        bad = gout.clone()
        bad[20, 30] = value
        gx, gw, gb = b.linear_backward(bad, x, w, preact=z, activation="gelu")
        rows, cols = [i for i in range(n) if i != 20], [i for i in range(m) if i != 30]
        assert torch.equal(gx[rows], clean[0][rows]) and torch.equal(gw[cols], clean[1][cols]) and torch.equal(gb[cols], clean[2][cols])
        assert not torch.isfinite(gx[20]).any() and not torch.isfinite(gw[30]).any() and not torch.isfinite(gb[30])


@pytest.mark.parametrize("m", [7, 256, 257, 2000])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 9000])
def test_every_share_of_rows_and_columns(b, n, m):
    """However rows and columns divide among CTAs: every row and column of a size of its own, between 2^-14 and 2^12."""
    gen = torch.Generator(device="cuda").manual_seed(n + m)
    k = 24
    rows, cols = (torch.exp2(torch.randint(-7, 7, (c,), generator=gen, device="cuda").float()) for c in (n, m))
    gout = (torch.randn(n, m, generator=gen, device="cuda") * rows[:, None] * cols).half()
    z, x, w = (matrix(*s, torch.float16, gen, scale=f) for s, f in (((n, m), 1.0), ((n, k), 1e-3), ((m, k), 1e-3)))
    check_gradient(b, gout, x, w, z, "silu", 0.5, of_the_largest)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["identity", "relu", "gelu"])
@pytest.mark.parametrize("n,k,m", [(15, 14, 9), (3, 300, 500), (300, 1, 40), (700, 130, 260)])
def test_every_choice_of_gradients(b, n, k, m, act, dtype):
    """Each of gx, gw and gbias with and without the others: the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    gout, z, x, w = (matrix(*s, dtype, gen) for s in ((n, m), (n, m), (n, k), (m, k)))
    every = b.linear_backward(gout, x, w, preact=z, activation=act, scale=0.5)
    for want in range(1, 8):
        got = b.linear_backward(gout, x, w, preact=z, activation=act, scale=0.5, want_x=bool(want & 1), want_w=bool(want & 2), want_bias=bool(want & 4))
        for i in range(3):
            assert torch.equal(got[i], every[i]) if want >> i & 1 else got[i] is None
