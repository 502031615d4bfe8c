"""Objective against cumulative coefficient updates under the three schedules the paper compares
(Section 5.1 and its convergence figure for the Lasso): the dynamic schedule of Algorithm 1 (priority draw +
rho filter), "static" (uniform draw + rho filter) and "random" (uniform draw, no dependency check).

    python -m paper_1312_5766_b200.compare_schedules [--workload c1] [--rounds N] [--every K] [--scale D] [--first-order LR]

Runs on a CUDA device through the library; prints one line per schedule and checkpoint.  The curves of the
paper's figure came from data that is not available; this regenerates their shape on the synthetic workloads.  With --first-order
a fourth curve follows, dense workloads only: full-gradient steps of AdamW with the L1 threshold, each an update of all J coefficients.
"""
from __future__ import annotations

import argparse

import torch

from . import binding, workloads as wl

SCHEDULES = {                      # name -> flags
    "priority": 0,
    "static": binding.FLAG_UNIFORM_DRAW,
    "random": binding.FLAG_UNIFORM_DRAW | binding.FLAG_NO_FILTER,
}


def trace(p: wl.LassoProblem, schedule: str, rounds: int, every: int, device="cuda", extra_flags: int = 0):
    """[(rounds done, cumulative updates, objective)] at round 0 and after every `every` rounds."""
    s = binding.StradsLasso.from_problem(p, device=device, flags=SCHEDULES[schedule] | extra_flags)
    out = [(0, 0, s.objective())]
    done = 0
    while done < rounds:
        n = min(every, rounds - done)
        s.run(n)
        done += n
        out.append((done, s.totals()["kept"], s.objective()))
    rc, bits = s.status()
    if rc != 0:
        raise binding.StradsError(rc, "strads_status")
    s.close()
    return out


def first_order_pass(x, y, beta, opt, step: int, lr: float, activation: str = "identity"):
    """One pass: residuals y - act(x beta^T) from the layer's epilogue, minus their product with x as the gradient, a step.  x [N, J]
    in either order, y [N, R], beta [R, J] (opt's parameter); returns the residuals it started from and the gradient."""
    resid = binding.linear_forward(x, beta, residual=y, activation=activation, scale=-1.0)
    _, grad, _ = binding.linear_backward(resid, x, beta, scale=-1.0, want_x=False, want_bias=False)
    opt.step([grad], lr=lr, step=step)
    return resid, grad


def first_order_trace(p: wl.LassoProblem, passes: int, every: int, lr: float, device="cuda"):
    """[(passes done, cumulative updates, objective)] as `trace`, under proximal AdamW on the whole gradient (dense problems)."""
    if p.layout != wl.DENSE:
        raise ValueError("the first-order curve needs a dense design")
    x, y = p.values.to(device)[:, : p.n_rows].t(), p.y.to(device)[:, None]
    beta = torch.zeros(1, p.n_cols, device=device)
    opt = binding.AdamW([beta], l1=p.lam)
    objective = lambda: 0.5 * float(binding.linear_forward(x, beta, residual=y, scale=-1.0).double().square().sum()) + \
        p.lam * float(beta.double().abs().sum())
    out = [(0, 0, objective())]
    for t in range(1, passes + 1):
        first_order_pass(x, y, beta, opt, t, lr)
        if t % every == 0 or t == passes:
            out.append((t, t * p.n_cols, objective()))
    rc, _ = binding.linear_status(x.device)
    if rc != 0:
        raise binding.StradsError(rc, "strads_linear_status")
    return out


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="c1")
    ap.add_argument("--scale", type=int, default=1, help="divide N, J, the true support, P' and P by this")
    ap.add_argument("--rounds", type=int, default=0, help="0: the workload's own round count (divided by --scale)")
    ap.add_argument("--every", type=int, default=0)
    ap.add_argument("--first-order", type=float, default=0.0, metavar="LR", help="also a curve of full-gradient AdamW steps of this size")
    args = ap.parse_args()
    cfg = dict(wl.scaled(args.workload, args.scale) if args.scale > 1 else wl.CONFIGS[args.workload], name=args.workload)
    p = wl.make_problem(cfg, seed=0, device="cuda" if torch.cuda.is_available() else "cpu")
    rounds = args.rounds or max(1, cfg["rounds"] // args.scale)
    every = args.every or max(1, rounds // 10)
    print(f"# {args.workload}/{args.scale}: N={p.n_rows} J={p.n_cols} P'={p.n_candidates} P={p.n_keep} rho={p.rho} lambda={p.lam:.6g}")
    print("schedule rounds updates objective")
    for name in SCHEDULES:
        for r, u, f in trace(p, name, rounds, every):
            print(f"{name} {r} {u} {f:.9g}")
    if args.first_order > 0:
        for r, u, f in first_order_trace(p, rounds, every, args.first_order):
            print(f"first_order {r} {u} {f:.9g}")


if __name__ == "__main__":
    main()
