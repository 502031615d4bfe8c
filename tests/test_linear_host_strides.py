"""Which strides strads_linear_* take for what they write, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding, build
    build.build()
    binding.load()
    return binding


TAKEN = [(5, 2), (7, 3), (6, 2), (1, 4), (2, 7), (3, 12), (1 << 61, 1), (1, 1 << 61), (1 << 61, 1 << 59)]
OVERLAPPING = [(4, 2), (2, 1), (1, 3), (2, 6), (3, 3), (0, 1), (1, 0), (1 << 61, 1 << 61), (1 << 61, 1 << 60)]


@pytest.mark.parametrize("rows_first", [True, False])
def test_strides_of_results(b, rows_first):
    """Four rows of three columns (of a call that then ends for want of workspace: -3): taken where no two elements share a place."""
    for strides, want in [(s, -3) for s in TAKEN] + [(s, -1) for s in OVERLAPPING]:
        n_rows, n_in, n_out = (300, 3, 4) if rows_first else (4, 3, 200)      # gw of 4 by 3, or gx of 4 by 3; gz goes through the workspace
        c = b.LinearConfig(type=0, activation=2, n_rows=n_rows, n_in=n_in, n_out=n_out, scale=1.0)
        c.x, c.x_row_stride, c.x_col_stride, c.w, c.w_row_stride, c.w_col_stride = 0x100000, n_in, 1, 0x200000, n_in, 1      # never dereferenced
        gout, z, m = b.Matrix(0x300000, n_out, 1), b.Matrix(0x400000, n_out, 1), b.Matrix(0x600000, *strides)
        gx, gw = (None, C.byref(m)) if rows_first else (C.byref(m), None)
        assert b.load().strads_linear_backward(C.byref(c), C.byref(gout), C.byref(z), gx, gw, None) == want, strides
