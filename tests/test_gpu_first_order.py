"""Layers, their gradients and steps together, as a first-order pass uses them, and the command that plots one beside the schedules."""
import subprocess
import sys

import pytest
import torch

from paper_1312_5766_b200 import workloads as wl

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.mark.parametrize("responses", [1, 3, 20, 200])
@pytest.mark.parametrize("activation", ["identity", "sigmoid"])
def test_passes_over_a_design(responses, activation):
    """Ten passes for several responses on a column-major design; every pass's residuals and gradient against 64 bits from the
    coefficients it started with, and its step against the formula from that gradient."""
    from paper_1312_5766_b200 import binding as b
    from paper_1312_5766_b200.compare_schedules import first_order_pass
    p = wl.make_problem(dict(kind="dense_iid", n_rows=301, n_cols=1000, n_true=20, lam_frac=0.05, n_candidates=10, n_keep=2, rho=0.1), seed=0)
    x = p.values.cuda()[:, : p.n_rows].t()
    gen = torch.Generator(device="cuda").manual_seed(0)
    y = torch.randn(p.n_rows, responses, generator=gen, device="cuda")
    y = (y > 0).float() if activation == "sigmoid" else y
    beta = torch.zeros(responses, p.n_cols, device="cuda")
    lam, lr, b1, b2, eps = 0.01, 1e-3, 0.9, 0.999, 1e-8
    opt = b.AdamW([beta], l1=lam)
    xd = x.to(F64)
    for t in range(1, 11):
        start = beta.to(F64)
        m0, v0 = (s[0].to(F64) for s in opt.moments())
        resid, grad = first_order_pass(x, y, beta, opt, t, lr, activation)
        z = xd @ start.t()
        want = y.to(F64) - (torch.sigmoid(z) if activation == "sigmoid" else z)
        # sums of 1,000 terms in 32 bits, and (sigmoid) a function good to 2^-20
        assert ((resid.to(F64) - want).abs() <= 1016 * 2.0 ** -24 * (xd.abs() @ start.abs().t()) + 2.0 ** -20 * (1 + want.abs())).all()
        r = resid.to(F64)
        assert ((grad.to(F64) + r.t() @ xd).abs() <= 317 * 2.0 ** -24 * (r.abs().t() @ xd.abs()) + 1e-37).all()
        g = grad.to(F64)
        m, v = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
        d = (v / (1 - b2 ** t)).sqrt() + eps
        q = start - lr * m / (1 - b1 ** t) / d
        q = q.sign() * (q.abs() - lr * lam / d).clamp(min=0)
        size = start.abs() + lr * (b1 * m0.abs() + (1 - b1) * g.abs()) / (1 - b1 ** t) / d + lr * lam / d
        assert ((beta.to(F64) - q).abs() <= 16 * 2.0 ** -24 * size).all(), t
    assert b.linear_status() == (0, 0)


def test_a_small_network_in_16_bits():
    """Two layers, bfloat16 with masters and 8-bit moments: the gradients that reach the steps against 64-bit autograd of the same network."""
    from paper_1312_5766_b200 import binding as b
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, k, h, m = 200, 96, 160, 40
    new = lambda *s, scale=1.0: (torch.randn(*s, generator=gen, device="cuda") * scale).bfloat16()
    x, target = new(n, k), new(n, m)
    params = [new(h, k, scale=0.1), new(h, scale=0.1), new(m, h, scale=0.08), new(m, scale=0.1)]
    masters = [p.float() for p in params]
    opt = b.AdamW(params, bits=8, masters=masters, weight_decay=0.01)
    for t in range(1, 4):
        w1, b1, w2, b2 = params
        a, z1 = b.linear_forward(x, w1, bias=b1, activation="gelu", want_preact=True)
        err = b.linear_forward(a, w2, bias=b2, residual=target, scale=-1.0)          # target - layer: minus the squared loss's gradient
        ga, gw2, gb2 = b.linear_backward(err, a, w2, scale=-1.0)
        _, gw1, gb1 = b.linear_backward(ga, x, w1, preact=z1, activation="gelu", want_x=False)
        leaves = [p.to(F64).requires_grad_(True) for p in params]
        hid = torch.nn.functional.gelu(x.to(F64) @ leaves[0].t() + leaves[1])
        (0.5 * (target.to(F64) - (hid @ leaves[2].t() + leaves[3])).square().sum()).backward()
        # each of the chain's five intermediate results is rounded to eps / 2 = 2^-8 of its value: in norm, no more than that much each
        for got, leaf in zip((gw1, gb1, gw2, gb2), leaves):
            assert (got.to(F64) - leaf.grad).norm() <= 6 * 2.0 ** -8 * leaf.grad.norm()
        before = [q.clone() for q in masters]
        opt.step([gw1, gb1, gw2, gb2], lr=1e-3, step=t)
        for p, q, o in zip(params, masters, before):
            assert torch.equal(p, q.bfloat16()) and not torch.equal(q, o) and (q - o).abs().max() <= 5e-3


def test_the_command_prints_the_curve():
    out = subprocess.run([sys.executable, "-m", "paper_1312_5766_b200.compare_schedules", "--workload", "c1", "--scale", "10", "--rounds", "20", "--every", "10",
                          "--first-order", "0.01"], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    rows = [r.split() for r in out.stdout.splitlines() if r.startswith("first_order")]
    assert [(int(r[1]), int(r[2])) for r in rows] == [(0, 0), (10, 10_000), (20, 20_000)]
    assert all(float(r[3]) > 0 for r in rows)


def test_sparse_designs_are_refused():
    from paper_1312_5766_b200 import compare_schedules as cs
    p = wl.make_problem(dict(kind="csc_uniform", n_rows=64, n_cols=100, n_true=1, lam_frac=0.1, nnz_col=2, n_candidates=10, n_keep=1, rho=0.1), seed=0)
    with pytest.raises(ValueError):
        cs.first_order_trace(p, 1, 1, 0.01)
