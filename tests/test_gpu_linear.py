"""Linear layers and their gradients against the formula in 64 bits.

Tolerances, element by element.  S is the sum of the magnitudes of an element's terms.  A sum of K terms held in 32 bits is off by at
most K 2^-24 S when every addition rounds to nearest, and where additions of 16 products at a time truncate (2^-23 of what has been
summed so far, K / 16 times) by less; the three 8-bit parts of a binary32 operand leave out 2^-24 of a product a few times over:
(K + 16) 2^-24 S covers either.  No activation's slope exceeds 1.13.  The function itself is good to 2^-20 of its value, and the
result is rounded to its type: eps / 2 relative, and half a subnormal step of binary16 (2^-25).  A 16-bit gradient's gz is rounded
to the type where the products read it: eps / 2 of S more.
"""
import math
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
F64 = torch.float64
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = ["identity", "relu", "sigmoid", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding
    return binding


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "sigmoid":
        return torch.special.expit(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(z * -math.sqrt(0.5))      # (1 + erf would lose what is small to binary64's own rounding)
    if act == "gelu_tanh":
        return z * torch.special.expit(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))      # (1 + tanh u) / 2 = sigma(2 u)
    return z * torch.special.expit(z) if act == "silu" else z


def slope64(z, act):
    if act == "identity":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(F64)
    z = z.clone().requires_grad_(True)
    act64(z, act).sum().backward()
    return z.grad.detach()


def matrix(rows, cols, dtype, gen, order="rows", scale=1.0, pad=0):
    """A matrix in the order of its rows or columns, contiguous or `pad` elements apart, with NaN in between."""
    r, c = (rows, cols) if order == "rows" else (cols, rows)
    t = torch.full((r, c + pad), float("nan"), dtype=dtype, device="cuda")
    v = t[:, pad:] if pad % 2 else t[:, :c]
    v.copy_(torch.randn(r, c, generator=gen, device="cuda") * scale)
    return v if order == "rows" else v.t()


def close(got, want, tol):
    d = (got.double() - want).abs()
    bad = ~(d <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, by up to {float((d / tol).nan_to_num(1e9).max()):.3g} times the tolerance"


def half_step(want, dtype):
    return torch.finfo(dtype).eps / 2 * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 1e-37)


def check_forward(b, x, w, bias, residual, act, scale, **kw):
    out, z = b.linear_forward(x, w, bias=bias, residual=residual, activation=act, scale=scale, want_preact=True, **kw)
    k = x.shape[1]
    xd, wd = x.to(F64), w.to(F64)
    z64 = xd @ wd.t()
    s = xd.abs() @ wd.abs().t()
    if bias is not None:
        z64, s = z64 + bias.to(F64), s + bias.to(F64).abs()
    summed = (k + 16) * 2.0 ** -24 * s
    close(z, z64, summed + half_step(z64.abs() + summed, x.dtype))
    a = scale * act64(z64, act)
    want = a if residual is None else residual.to(F64) + a
    tol = 1.13 * abs(scale) * summed + 2.0 ** -20 * a.abs()
    close(out, want, tol + half_step(want.abs() + tol, x.dtype))
    return out, z


def check_backward(b, gout, x, w, z, act, scale, **kw):
    gx, gw, gb = b.linear_backward(gout, x, w, preact=z, activation=act, scale=scale, **kw)
    u = 0.0 if x.dtype == torch.float32 else torch.finfo(x.dtype).eps / 2
    small = 2.0 ** -25 if x.dtype == torch.float16 else 0.0
    gz = scale * gout.to(F64) * (slope64(z.to(F64), act) if z is not None else 1.0)
    # the slope's own error: 2^-20 of the largest slope
    e = gz.abs() * (u + 2.0 ** -20) + 2.0 ** -20 * abs(scale) * gout.to(F64).abs() + small
    (n, k), m = x.shape, w.shape[0]
    for got, want, mag, err, terms in ((gx, lambda: gz @ w.to(F64), lambda: gz.abs() @ w.to(F64).abs(), lambda: e @ w.to(F64).abs(), m),
                                       (gw, lambda: gz.t() @ x.to(F64), lambda: gz.abs().t() @ x.to(F64).abs(), lambda: e.t() @ x.to(F64).abs(), n),
                                       (gb, lambda: gz.sum(0), lambda: gz.abs().sum(0), lambda: e.sum(0), n)):
        if got is not None:
            v = want()
            tol = (terms + 16) * 2.0 ** -24 * mag() + err()
            close(got, v, tol + half_step(v.abs() + tol, x.dtype))
    return gx, gw, gb


SHAPES = [(1, 1, 1), (1, 7, 513), (1, 1000, 1), (2, 64, 200), (3, 1001, 129), (7, 4096, 256), (8, 513, 8), (9, 100, 300), (16, 128, 128), (17, 1000, 33),
          (33, 5, 1000), (64, 2048, 64), (100, 300, 20), (128, 64, 128), (129, 257, 131), (255, 512, 256), (300, 1001, 517), (1000, 3, 2),
          (1000, 2000, 1), (500, 8, 3000), (257, 1024, 2049)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)), ids=lambda i: "x".join(map(str, SHAPES[i])))
def test_forward(b, i, dtype):
    n, k, m = SHAPES[i]
    for turn in range(4):                                # orders of x and w
        gen = torch.Generator(device="cuda").manual_seed(100 * i + turn)
        x = matrix(n, k, dtype, gen, "rows" if turn % 2 == 0 else "cols")
        w = matrix(m, k, dtype, gen, "rows" if turn < 2 else "cols", scale=k ** -0.5)
        bias = torch.randn(m, generator=gen, device="cuda").to(dtype) if (i + turn) % 3 else None
        residual = matrix(n, m, dtype, gen) if (i + turn) % 2 else None
        check_forward(b, x, w, bias, residual, ACTS[(i + turn) % 6], (1.0, -1.0, 0.5)[(i + turn) % 3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("i", range(len(SHAPES)), ids=lambda i: "x".join(map(str, SHAPES[i])))
def test_backward(b, i, dtype):
    n, k, m = SHAPES[i]
    for turn in range(4):
        gen = torch.Generator(device="cuda").manual_seed(100 * i + turn)
        x = matrix(n, k, dtype, gen, "rows" if turn % 2 == 0 else "cols")
        w = matrix(m, k, dtype, gen, "rows" if turn < 2 else "cols", scale=k ** -0.5)
        act = ACTS[(i + turn) % 6]
        z = matrix(n, m, dtype, gen) if act != "identity" else None
        g = check_backward(b, matrix(n, m, dtype, gen), x, w, z, act, (1.0, -1.0, 0.5)[(i + turn) % 3])
        assert g[0].stride() == x.stride() or min(x.shape) == 1
        assert g[1].stride() == w.stride() or min(w.shape) == 1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_every_activation_over_its_range(b, act, dtype):
    """z from far below to far above: x is z, w is 1."""
    z = torch.cat([torch.linspace(-90, 90, 4001), torch.linspace(-1, 1, 2001), torch.tensor([0.0, -0.0, 1e-6, -1e-6, 60.0, -60.0])])
    x = z.to(dtype).cuda()[:, None]
    w = torch.ones(1, 1, dtype=dtype, device="cuda")
    out, keep = b.linear_forward(x, w, activation=act, want_preact=True)
    assert torch.equal(keep, x)                          # a sum of one product of 1
    want = act64(x.to(F64), act)
    # relative to the value even where it is small: nothing cancels.  The argument of exp carries 2^-22 of itself, so its
    # value |argument| 2^-22: for the tanh form that is 1.6 (|z| + 0.045 |z|^3).  A sigma or Phi below 2^-126 may be lost to the range of binary32, and
    # with it z times that, at most 90 2^-126 < 2^-119
    arg = {"gelu_tanh": lambda t: 1.6 * (t + 0.045 * t ** 3), "gelu": lambda t: t * t / 2}.get(act, lambda t: t)(x.to(F64).abs())
    tol = want.abs() * (2.0 ** -20 + arg.clamp(max=120) * 2.0 ** -21) + 2.0 ** -119
    close(out, want, tol + half_step(want.abs() + tol, dtype))
    g = torch.ones_like(x)
    gx, _, _ = b.linear_backward(g, x, w, preact=x, activation=act)
    want = slope64(x.to(F64), act)
    u = 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2
    tol = (u + 2.0 ** -20) * want.abs() + 2.0 ** -20 + (2.0 ** -25 if dtype == torch.float16 else 0)
    close(gx, want, tol + half_step(want.abs() + tol, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(3, 50, 70), (140, 200, 130), (257, 600, 300)])
@pytest.mark.parametrize("pad", [1, 2, 3, 8, 64])
def test_padded_rows_and_odd_offsets(b, dtype, shape, pad):
    """Operands that are parts of larger matrices, at offsets that divide by nothing, NaN all around; outputs likewise."""
    n, k, m = shape
    gen = torch.Generator(device="cuda").manual_seed(pad)
    for ox, ow in (("rows", "rows"), ("cols", "cols")):
        x, w = matrix(n, k, dtype, gen, ox, pad=pad), matrix(m, k, dtype, gen, ow, scale=k ** -0.5, pad=pad)
        residual, z = matrix(n, m, dtype, gen, "rows", pad=pad), matrix(n, m, dtype, gen, "cols", pad=pad)
        whole = torch.full((n + 2, m + pad + 2), 77.0, dtype=dtype, device="cuda")
        keep = whole.clone()
        bias = torch.randn(m + 1, generator=gen, device="cuda").to(dtype)[1:]
        check_forward(b, x, w, bias, residual, "gelu", -0.5, out=whole[1:-1, 1:1 + m], preact=keep[1:-1, 1:1 + m])
        for t in (whole, keep):
            t[1:-1, 1:1 + m] = 77.0
            assert (t == 77.0).all()
        gx, gw = (torch.full((r + 2, c + pad + 2), 77.0, dtype=dtype, device="cuda") for r, c in ((n, k), (m, k)))
        check_backward(b, matrix(n, m, dtype, gen, "rows", pad=pad), x, w, z, "silu", 1.0, grad_x=gx[1:-1, 1:1 + k], grad_w=gw[1:-1, 1:1 + k])
        gx[1:-1, 1:1 + k] = 77.0
        gw[1:-1, 1:1 + k] = 77.0
        assert (gx == 77.0).all() and (gw == 77.0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_repeated_and_strided_operands(b, dtype):
    gen = torch.Generator(device="cuda").manual_seed(0)
    for n, k, m in ((5, 40, 30), (150, 200, 260)):
        y = torch.randn(n, 1, generator=gen, device="cuda").to(dtype)
        w = matrix(m, k, dtype, gen, scale=k ** -0.5)
        x = matrix(n, k, dtype, gen)
        check_forward(b, x, w, None, y.expand(n, m), "sigmoid", -1.0)                     # one y for every response
        check_forward(b, x[:1].expand(n, k), w, None, None, "identity", 1.0)              # rows repeated
        check_forward(b, matrix(2 * n, 3 * k, dtype, gen)[::2, ::3], w, None, None, "relu", 1.0)
        check_forward(b, x, matrix(m, 2 * k, dtype, gen)[:, ::2], None, None, "relu", 1.0)
        check_backward(b, y.expand(n, m), x, w, matrix(n, 2 * m, dtype, gen)[:, ::2], "gelu", 1.0)
        # results in the order of columns, and two elements apart
        check_forward(b, x, w, None, None, "relu", 1.0, out=torch.empty(m, n, dtype=dtype, device="cuda").t())
        check_forward(b, x, w, None, None, "relu", 1.0, out=torch.empty(n, 2 * m, dtype=dtype, device="cuda")[:, ::2])
        check_backward(b, matrix(n, m, dtype, gen), x, w, None, "identity", 1.0, grad_w=torch.empty(k, m, dtype=dtype, device="cuda").t(),
                       grad_x=torch.empty(n, 2 * k, dtype=dtype, device="cuda")[:, ::2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 6, 40, 300])
def test_what_is_not_finite_stays_in_its_row(b, dtype, n):
    gen = torch.Generator(device="cuda").manual_seed(n)
    k, m = 300, 200
    x, w = matrix(n, k, dtype, gen), matrix(m, k, dtype, gen, scale=k ** -0.5)
    clean = b.linear_forward(x, w, activation="relu")
    for value in (float("nan"), float("inf"), float("-inf")):
        bad = x.clone()
        bad[n // 2, 17] = value
        got = b.linear_forward(bad, w)
        others = [r for r in range(n) if r != n // 2]
        assert torch.equal(b.linear_forward(bad, w, activation="relu")[others], clean[others])
        assert not torch.isfinite(got[n // 2]).any()
        ww = w.clone()
        ww[11, k - 1] = value
        got = b.linear_forward(x, ww, activation="relu")
        assert torch.equal(torch.cat([got[:, :11], got[:, 12:]], 1), torch.cat([clean[:, :11], clean[:, 12:]], 1))
        gx, gw, gb = b.linear_backward(b.linear_forward(bad, w), x, w)
        assert torch.isfinite(gx[others]).all() and not torch.isfinite(gb).any()


@pytest.mark.parametrize("tiles,blocks", [(1, 1), (1, 3), (1, 40), (2, 9), (5, 31), (147, 2), (148, 3), (149, 3), (150, 2), (300, 2), (37, 16)])
@pytest.mark.parametrize("order", ["rows", "cols"])
def test_shares_of_tiles(b, tiles, blocks, order):
    """binary32 with few rows on one side: tiles of 128 rows by blocks of 64 k, however they divide among the CTAs; NaN in the memory that
    the partial sums get."""
    n, k = 128 * tiles - 5, 64 * blocks - 3
    gen = torch.Generator(device="cuda").manual_seed(tiles)
    whole = torch.full((k, n + 5) if order == "cols" else (n, k + 3), float("nan"), device="cuda")      # runs that start on 16 bytes, NaN behind them
    x = whole[:, :n].t() if order == "cols" else whole[:, :k]
    x.copy_(torch.randn(n, k, generator=gen, device="cuda"))
    for m in (7, 33, 50):
        junk = torch.full((64 << 20,), float("nan"), device="cuda")
        del junk
        check_forward(b, x, matrix(m, k, torch.float32, gen, scale=k ** -0.5), None, None, "identity", 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(b, dtype):
    x, w = torch.empty(0, 30, dtype=dtype, device="cuda"), torch.randn(20, 30, device="cuda").to(dtype)
    out, z = b.linear_forward(x, w, want_preact=True, activation="gelu")
    assert out.shape == z.shape == (0, 20)
    gx, gw, gb = b.linear_backward(torch.empty(0, 20, dtype=dtype, device="cuda"), x, w, preact=z, activation="gelu", grad_w=torch.ones_like(w),
                                   grad_bias=torch.ones(20, dtype=dtype, device="cuda"))
    assert gx.shape == (0, 30) and not gw.any() and not gb.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 5, 200])
def test_out_may_be_the_residual(b, dtype, n):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, w, r = matrix(n, 256, dtype, gen), matrix(144, 256, dtype, gen, scale=0.06), matrix(n, 144, dtype, gen)
    want = b.linear_forward(x, w, residual=r, activation="silu", scale=0.5)
    got = b.linear_forward(x, w, residual=r, activation="silu", scale=0.5, out=r)
    assert got is r and torch.equal(got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 24, 600])
def test_captured_and_replayed(b, dtype, n):
    """Two graphs, replayed in turn and on new inputs, and calls beside them on another stream: the bits of direct calls."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, w, g = matrix(n, 500, dtype, gen), matrix(300, 500, dtype, gen, scale=0.05), matrix(n, 300, dtype, gen)

    def once():
        out, z = b.linear_forward(x, w, activation="gelu", want_preact=True)
        return [out, *b.linear_backward(g, x, w, preact=z, activation="gelu")]

    once()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(once())
        graphs.append(graph)
    side = torch.cuda.Stream()
    for turn in range(3):
        x.copy_(torch.randn(n, 500, generator=gen, device="cuda"))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            beside = once()
        for graph in graphs:
            graph.replay()
        torch.cuda.current_stream().wait_stream(side)
        want = once()
        for got in outs + [beside]:
            assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 2000, 600), (30, 2000, 600), (700, 900, 800)])
def test_same_bits_every_time(b, dtype, shape):
    n, k, m = shape
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, g = matrix(n, k, dtype, gen), matrix(m, k, dtype, gen), matrix(n, m, dtype, gen)
    runs = [[b.linear_forward(x, w), *b.linear_backward(g, x, w)] for _ in range(3)]
    assert all(torch.equal(p, q) for r in runs[1:] for p, q in zip(r, runs[0]))


def test_offsets_past_32_bits(b):
    """A weight of 2.8 G elements, by one row, by twenty, and its gradient; spots of the results against 64 bits."""
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    m, k = 70_000, 40_000
    gen = torch.Generator(device="cuda").manual_seed(9)
    w = torch.empty(m, k, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    x = matrix(20, k, torch.bfloat16, gen)
    rows = torch.tensor([0, 1, 53_686, 53_687, 53_688, 69_998, 69_999], device="cuda")      # 2^31 / k = 53,687.1
    for n in (1, 20):
        out = b.linear_forward(x[:n], w)
        z64 = x[:n].to(F64) @ w[rows].to(F64).t()
        s = (k + 16) * 2.0 ** -24 * (x[:n].to(F64).abs() @ w[rows].to(F64).abs().t())
        close(out[:, rows], z64, s + half_step(z64.abs() + s, torch.bfloat16))
        g = matrix(n, m, torch.bfloat16, gen)
        _, gw, gb = b.linear_backward(g, x[:n], w, want_x=False, grad_w=w.new_empty(m, k))
        want = g[:, rows].to(F64).t() @ x[:n].to(F64)
        tol = (n + 16) * 2.0 ** -24 * (g[:, rows].to(F64).abs().t() @ x[:n].to(F64).abs())
        close(gw[rows], want, tol + half_step(want.abs() + tol, torch.bfloat16))
        # the same weight in the order of its columns: rows of x run through memory
        gt, xt = w.view(-1)[: n * m].view(m, n).t(), w.view(-1)[-n * k:].view(n, k)
        out = b.linear_forward(gt, xt.new_ones(3, m))
        assert torch.isfinite(out).all()
        del gw


@pytest.mark.parametrize("n", [1, 40])
def test_the_first_call_of_a_process_may_be_captured(n):
    code = f"""
import sys, torch
from paper_1312_5766_b200 import binding as b
x, w = torch.randn({n}, 512, device="cuda").bfloat16(), torch.randn(256, 512, device="cuda").bfloat16()
p, g = torch.randn(1000, device="cuda"), torch.randn(1000, device="cuda")
opt = b.AdamW([p])
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = b.linear_forward(x, w, activation="gelu")
    grads = b.linear_backward(out, x, w)
    opt.step([g], step=1)
q = p.clone()
graph.replay()
torch.cuda.synchronize()
assert torch.equal(out, b.linear_forward(x, w, activation="gelu"))
assert all(torch.equal(s, t) for s, t in zip(grads, b.linear_backward(out, x, w)))
assert not torch.equal(p, q)
"""
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


def test_gradients_against_differences(b):
    """d/dt F(p + t d) at t = 0 by central differences of the float32 layer, F = sum of c * out.  With steps of 1/64 the third
    derivative's term is (1/64)^2 / 6 F''' ~ 4e-5 F''', and 32-bit outputs, good to 2^-20 of the sum of magnitudes, leave
    2^-20 * 64 of it: both are below 1e-3 of the sum of the magnitudes of the gradient's terms."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, k, m = 19, 40, 23
    for act in ("sigmoid", "gelu", "gelu_tanh", "silu"):
        p = [matrix(n, k, torch.float32, gen), matrix(m, k, torch.float32, gen, scale=k ** -0.5), torch.randn(m, generator=gen, device="cuda")]
        c = matrix(n, m, torch.float32, gen)
        _, z = b.linear_forward(p[0], p[1], bias=p[2], activation=act, scale=0.5, want_preact=True)
        grads = b.linear_backward(c, p[0], p[1], preact=z, activation=act, scale=0.5)
        for i in range(3):
            d = torch.randn(p[i].shape, generator=gen, device="cuda")
            f = []
            for t in (1 / 64, -1 / 64):
                q = list(p)
                q[i] = p[i] + t * d
                f.append(float((c.double() * b.linear_forward(q[0], q[1], bias=q[2], activation=act, scale=0.5).double()).sum()))
            terms = grads[i].double() * d.double()
            assert abs((f[0] - f[1]) * 32 - float(terms.sum())) <= 1e-3 * float(terms.abs().sum())


STALLS = [(300, 512, 256, torch.bfloat16, "rows"), (40, 2000, 300, torch.float16, "cols"), (4096, 512, 4096, torch.bfloat16, "rows"), (300, 900, 200, torch.float32, "rows"),
          (1000, 2000, 1, torch.float32, "cols"), (1000, 2000, 3, torch.bfloat16, "cols"), (900, 1000, 20, torch.float32, "cols"), (900, 1000, 40, torch.float32, "rows")]


@pytest.mark.parametrize("n,k,m,dtype,order", STALLS, ids=str)
def test_a_wait_that_runs_out_is_reported(b, n, k, m, dtype, order):
    """Operand loads withheld, in every kernel that waits for some: the call ends after milliseconds, the status says so once, and the next
    call is right."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, w = matrix(n, k, dtype, gen, order), matrix(m, k, dtype, gen)
    assert b.linear_status() == (0, 0)
    want = b.linear_forward(x, w)
    b.linear_forward(x, w, flags=b.LINEAR_FLAG_STALL)
    assert b.linear_status() == (-6, 4)
    assert b.linear_status() == (0, 0)
    assert torch.equal(b.linear_forward(x, w), want)
    assert b.linear_status() == (0, 0)


def test_the_binding_refuses(b):
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    for call in (lambda: b.linear_forward(x, w[:, :7]), lambda: b.linear_forward(x, w.cpu()), lambda: b.linear_forward(x, w, bias=torch.zeros(4, device="cuda")),
                 lambda: b.linear_forward(x, w, activation="tanh"), lambda: b.linear_forward(x, w, residual=torch.zeros(3, 4, device="cuda")),
                 lambda: b.linear_backward(torch.zeros(4, 3, device="cuda"), x, w, activation="relu"),
                 lambda: b.linear_backward(torch.zeros(3, 4, device="cuda"), x, w)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: b.linear_forward(x, w.half()), lambda: b.linear_forward(x.double(), w.double()),
                 lambda: b.linear_forward(x, w, bias=torch.zeros(3, dtype=torch.float16, device="cuda"))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: b.linear_forward(x, w, scale=float("nan")), lambda: b.linear_forward(x, w, flags=2),
                 lambda: b.linear_forward(x, w, out=torch.zeros(1, 3, device="cuda").expand(4, 3))):
        with pytest.raises(b.StradsError):
            call()


# results of 74 tiles of 256 x 256 and more, which pairs of CTAs form: last tiles of 1, 8, 10, 36 and 255 rows or columns, results that TMA can address and
# (2,570) cannot, one block of k and several
PAIRS = [(2305, 70, 2568), (2340, 1, 2570), (2340, 200, 2568), (2559, 130, 2312), (4097, 64, 1288)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("i", range(len(PAIRS)), ids=lambda i: "x".join(map(str, PAIRS[i])))
def test_tiles_of_pairs(b, i, dtype):
    n, k, m = PAIRS[i]
    for turn, act in enumerate(ACTS):
        gen = torch.Generator(device="cuda").manual_seed(1000 + 10 * i + turn)
        x = matrix(n, k, dtype, gen, "rows" if turn % 2 == 0 else "cols")
        w = matrix(m, k, dtype, gen, "cols" if turn % 3 == 0 else "rows", scale=k ** -0.5)
        bias = torch.randn(m, generator=gen, device="cuda").to(dtype) if turn % 3 else None
        residual = matrix(n, m, dtype, gen, "cols" if turn == 4 else "rows") if turn != 1 else None
        out = matrix(n, m, dtype, gen, "cols" if turn in (2, 4) else "rows", pad=(0, 8)[turn == 5])
        check_forward(b, x, w, bias, residual, act, (1.0, -1.0, 0.5)[turn % 3], out=out)
        edge = out.as_strided((n, 8), (m + 8, 1), out.storage_offset() + m) if turn == 5 else None
        assert edge is None or torch.isnan(edge).all()   # what lies between the rows stays
        # the same tiles as a gradient: gx is n x m
        gout, v = matrix(n, k, dtype, gen), matrix(k, m, dtype, gen, "cols" if turn % 2 else "rows", scale=k ** -0.5)
        z = matrix(n, k, dtype, gen) if act != "identity" else None
        check_backward(b, gout, matrix(n, m, dtype, gen), v, z, act, 0.5)


def test_threads_on_streams_of_their_own(b):
    """Four threads at once, each with a stream, calls and workspaces of its own: the bits of the same calls one after another."""
    import threading
    gen = torch.Generator(device="cuda").manual_seed(5)
    cases = [(1000, 500, 20, torch.float32), (24, 900, 700, torch.bfloat16), (2340, 100, 2568, torch.float16), (333, 1001, 517, torch.float32)]
    inputs = [(matrix(n, k, t, gen), matrix(m, k, t, gen, scale=0.05), matrix(n, m, t, gen)) for n, k, m, t in cases]

    def once(x, w, g):
        out, z = b.linear_forward(x, w, activation="silu", want_preact=True)
        return [out, *b.linear_backward(g, x, w, preact=z, activation="silu")]

    want = [once(*v) for v in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got = once(*inputs[i])
                    if not all(torch.equal(p, q) for p, q in zip(got, want[i])):
                        wrong.append(i)
        except Exception as e:
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and b.linear_status() == (0, 0)
