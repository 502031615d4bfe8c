"""Linear layers over long k, one-signed, and over operands of more than 2^31 elements in either order."""
import pytest
import torch

from test_gpu_linear import ACTS, F64, b, check_backward, check_forward, close, half_step, matrix  # noqa: F401

pytestmark = pytest.mark.gpu


# narrow tiles, 128 columns, pairs of CTAs; CTAs that share a tile and that do not; runs of 4,096 terms with and without a remainder
LONG = [(torch.float16, 5, 1 << 21, 300), (torch.float16, 40, 1 << 21, 100), (torch.float16, 140, 1 << 21, 130), (torch.float16, 140, 70_001, 130),
        (torch.float16, 2309, 8_192, 2310), (torch.float16, 2309, 8_200, 2310), (torch.float16, 2309, 12_613, 2310), (torch.float16, 2309, 1 << 17, 2310),
        (torch.bfloat16, 40, 1 << 22, 100), (torch.bfloat16, 140, 1 << 22, 130), (torch.bfloat16, 2309, 100_003, 2310), (torch.bfloat16, 2309, 1 << 18, 2310)]


@pytest.mark.parametrize("dtype,n,k,m", LONG, ids=str)
@pytest.mark.parametrize("order", ["rows", "cols"])
def test_one_signed_sums_over_long_k(b, dtype, n, k, m, order):
    """Products of one sign, the sum without its rounding (the difference to its rounding, as a residual).  The tensor cores' additions truncate, 16 products at a time: 256 of
    them to a run of 4,096 terms, or 512 where one accumulator holds up to 8,192 (binary16); each loses 1.6 2^-23 of the sum so far on average (measured), which is half the
    run's: 5e-5.  A tenth of bfloat16's half step, 2^-8, where that type's takes up to 65,536.  The runs are added with rounding, up to 2^10 of them, 2^-25 each: 2^-16 at most."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    new = lambda rows: (torch.rand((rows, k) if order == "rows" else (k, rows), generator=gen, device="cuda", dtype=torch.float32).add_(1.0).mul_(2.0 ** -6)).to(dtype)
    x, w = new(n), new(m)
    if order == "cols":
        x, w = x.t(), w.t()
    rows, cols = [r % n for r in (0, 1, n // 2, n - 1)], [c % m for c in (0, 1, 17, m // 2, m - 1)]
    want = torch.stack([torch.stack([(x[r].to(F64) * w[c].to(F64)).sum() for c in cols]) for r in rows])
    out = b.linear_forward(x, w)
    rest = b.linear_forward(x, w, residual=out, scale=-1.0)[rows][:, cols]
    cut = (5e-5 if dtype == torch.float16 else 0.1 * 2.0 ** -8) + 2.0 ** -16
    close(out[rows][:, cols].double() - rest.double(), want, cut * want + half_step(rest.double(), dtype))
    # the same sums as a gradient over k rows
    _, gw, _ = b.linear_backward(x.t(), w.t(), x.new_empty(n, m), want_x=False, want_bias=False)
    close(gw[rows][:, cols], want, cut * want + half_step(want * (1 + cut), dtype))


@pytest.mark.parametrize("n,m", [(20, 50), (33, 300), (140, 1000), (2309, 2312)])
@pytest.mark.parametrize("turn", range(6))
def test_epilogues_of_kept_sums(b, n, m, turn):
    """Everything in the epilogue behind 75,000 terms of binary16, with results that TMA writes and others, and their gradient."""
    k, t, gen = 75_000, torch.float16, torch.Generator(device="cuda").manual_seed(n + turn)
    x, w = matrix(n, k, t, gen, "cols" if turn == 1 else "rows"), matrix(m, k, t, gen, scale=k ** -0.5)
    bias = torch.randn(m, generator=gen, device="cuda").to(t) if turn % 3 else None
    residual = matrix(n, m, t, gen, "cols" if turn == 4 else "rows") if turn % 2 else None
    out = matrix(n, m, t, gen, "cols" if turn == 2 else "rows", pad=(0, 8, 3)[turn % 3])
    check_forward(b, x, w, bias, residual, ACTS[turn], (1.0, -1.0, 0.5)[turn % 3], out=out)
    if n < 2000:                                         # gw sums over 75,000 rows
        z = matrix(k, n, t, gen) if turn else None
        check_backward(b, matrix(k, n, t, gen), matrix(k, m, t, gen), matrix(n, m, t, gen), z, ACTS[turn], 2.0 ** -10, want_x=False)


@pytest.mark.parametrize("n,m", [(20, 50), (140, 1000), (2309, 2312)])
def test_a_wait_that_runs_out_with_kept_sums(b, n, m):
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, w = matrix(n, 75_000, torch.float16, gen), matrix(m, 75_000, torch.float16, gen)
    assert b.linear_status() == (0, 0)
    want = b.linear_forward(x, w)
    b.linear_forward(x, w, flags=b.LINEAR_FLAG_STALL)
    assert b.linear_status() == (-6, 4)
    assert torch.equal(b.linear_forward(x, w), want) and b.linear_status() == (0, 0)


@pytest.mark.parametrize("n,m", [(3, 300), (20, 1000), (200, 300)])
def test_one_signed_sums_in_32_bits(b, n, m):
    """100,000 terms of one sign, binary32: errors do not grow with k.  Runs of at most 256 terms lose 2^-23 of the sum so far in each of up to 24 additions of products of
    planes a block of 64: below 2^-20; some 1,600 runs added with rounding, 2^-25 each, independent: 40 of them in the mean, below 2^-19.  An accumulator that
    is never emptied is off by 2e-5, 2^-15.6."""
    k = 100_000
    gen = torch.Generator(device="cuda").manual_seed(n)
    for order in ("rows", "cols"):
        new = lambda rows: torch.rand((rows, k) if order == "rows" else (k, rows), generator=gen, device="cuda").add_(0.5)
        x, w = new(n), new(m)
        if order == "cols":
            x, w = x.t(), w.t()
        want = x.to(F64) @ w.to(F64).t()
        close(b.linear_forward(x, w), want, 2.0 ** -18 * want)


@pytest.mark.parametrize("n", [1, 3, 20])
def test_columns_past_32_bits(b, n):
    """2.8 G elements of bfloat16 in the order of their columns, against all rows, and spots of the results beside element 2^31 against 64 bits."""
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    m, k = 40_000, 70_000
    gen = torch.Generator(device="cuda").manual_seed(9)
    w = torch.empty(k, m, dtype=torch.bfloat16, device="cuda").normal_(generator=gen).t()
    x = matrix(n, k, torch.bfloat16, gen)
    at = torch.tensor([0, 1, 127, 128, 20_000, m - 2, m - 1], device="cuda")
    out = b.linear_forward(x, w)
    xd, wd = x.to(F64), w[at].to(F64)
    s = (k + 16) * 2.0 ** -24 * (xd.abs() @ wd.abs().t())
    close(out[:, at], xd @ wd.t(), s + half_step((xd @ wd.t()).abs() + s, torch.bfloat16))
    # gx reads the same matrix along its rows, gw writes one like it
    g = matrix(n, m, torch.bfloat16, gen)
    rows = torch.tensor([0, 1, 53_686, 53_687, 53_688, k - 1], device="cuda")      # 2^31 / m = 53,687.1
    gx, gw, _ = b.linear_backward(g, x, w, want_bias=False)
    assert gw.stride() == w.stride()
    wd, gd = w[:, rows].to(F64), g.to(F64)
    s = (m + 16) * 2.0 ** -24 * (gd.abs() @ wd.abs())
    close(gx[:, rows], gd @ wd, s + half_step((gd @ wd).abs() + s, torch.bfloat16))
    want = gd.t() @ x[:, rows].to(F64)
    s = (n + 16) * 2.0 ** -24 * (gd.abs().t() @ x[:, rows].to(F64).abs())
    close(gw[:, rows], want, s + half_step(want.abs() + s, torch.bfloat16))


@pytest.mark.parametrize("order", ["rows", "cols"])
@pytest.mark.parametrize("n", [1, 20])
def test_binary32_past_32_bits(b, n, order):
    """The same for 2.4 G elements of binary32, streamed and split on the way."""
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    m, k = (60_000, 40_000) if order == "rows" else (40_000, 60_000)
    gen = torch.Generator(device="cuda").manual_seed(10)
    w = torch.empty(60_000, 40_000, device="cuda").normal_(generator=gen)
    w = w if order == "rows" else w.t()
    x, g = matrix(n, k, torch.float32, gen), matrix(n, m, torch.float32, gen)
    near = [53_686, 53_687, 53_688]                      # 2^31 / 40,000 = 53,687.1
    at = torch.tensor([0, 1, m // 2, m - 1] + (near if order == "rows" else []), device="cuda")
    rows = torch.tensor([0, 1, k // 2, k - 1] + (near if order == "cols" else []), device="cuda")
    xd, gd = x.to(F64), g.to(F64)
    wd = w[at].to(F64)
    s = (k + 16) * 2.0 ** -24 * (xd.abs() @ wd.abs().t())
    close(b.linear_forward(x, w)[:, at], xd @ wd.t(), s + half_step((xd @ wd.t()).abs() + s, torch.float32))
    gx, _, _ = b.linear_backward(g, x, w, want_w=False, want_bias=False)
    wd = w[:, rows].to(F64)
    s = (m + 16) * 2.0 ** -24 * (gd.abs() @ wd.abs())
    close(gx[:, rows], gd @ wd, s + half_step((gd @ wd).abs() + s, torch.float32))
