"""strads_linear_*: what they refuse, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_1312_5766_b200 import binding, build
    build.build()
    binding.load()
    return binding


def _config(b, **kw):
    c = b.LinearConfig(type=1, activation=3, n_rows=100, n_in=200, n_out=300, scale=1.0)
    c.x, c.x_row_stride, c.x_col_stride, c.w, c.w_row_stride, c.w_col_stride = 0x100000, 200, 1, 0x200000, 200, 1      # never dereferenced
    c.workspace, c.workspace_bytes = 0x10000000, 1 << 40
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _call(b, c, which, out=None, bias=None, **kw):
    lib = b.load()
    m = lambda rows, cols, at: b.Matrix(at, cols, 1)
    ref = lambda x: None if x is None else C.byref(x)
    if which == "forward":
        out = m(100, 300, 0x300000) if out is None else out
        return lib.strads_linear_forward(C.byref(c), bias, ref(kw.get("residual")), ref(out), ref(kw.get("preact")))
    gx = kw.get("gx", m(100, 200, 0x500000))
    return lib.strads_linear_backward(C.byref(c), ref(kw.get("gout", m(100, 300, 0x300000))), ref(kw.get("preact", m(100, 300, 0x400000))),
                                      ref(gx), ref(kw.get("gw")), bias)


CONFIGS = [dict(type=3), dict(type=-1), dict(activation=6), dict(activation=-1), dict(n_rows=-1), dict(n_in=0), dict(n_out=0),
           dict(scale=float("nan")), dict(scale=float("inf")), dict(flags=2), dict(workspace=0x10000010)]


@pytest.mark.parametrize("which", ["forward", "backward"])
@pytest.mark.parametrize("kw", CONFIGS, ids=str)
def test_bad_configurations(b, kw, which):
    if "workspace" in kw:                                # binary32 operands go through the workspace
        kw = dict(kw, type=0, n_rows=1000, n_in=1000, n_out=1000)
    assert _call(b, _config(b, **kw), which) == -1


@pytest.mark.parametrize("which", ["forward", "backward"])
def test_bad_operands(b, which):
    for x in (b.Matrix(None, 200, 1), b.Matrix(0x100001, 200, 1), b.Matrix(0x100000, -200, 1), b.Matrix(0x100000, 200, -1)):
        for side in "xw":
            assert _call(b, _config(b, **{side: x.data, side + "_row_stride": x.row_stride, side + "_col_stride": x.col_stride}), which) == -1
    for n in ("n_rows", "n_in", "n_out"):
        assert _call(b, _config(b, **{n: (1 << 30) + 1}), which) == -7


def test_bad_outputs(b):
    # null, misaligned, overlapping itself
    for out in (b.Matrix(None, 300, 1), b.Matrix(0x300001, 300, 1), b.Matrix(0x300000, 0, 1), b.Matrix(0x300000, 299, 1),
                b.Matrix(0x300000, 300, 0), b.Matrix(0x300000, 1, 99), b.Matrix(0x300000, 300, 2)):
        assert _call(b, _config(b), "forward", out=out) == -1
        assert _call(b, _config(b), "forward", preact=out) == -1
    for gx in (b.Matrix(None, 200, 1), b.Matrix(0x300000, 199, 1), b.Matrix(0x300000, 1, 99)):
        assert _call(b, _config(b), "backward", gx=gx) == -1
    assert _call(b, _config(b), "backward", gw=b.Matrix(0x300000, 0, 1)) == -1
    assert _call(b, _config(b), "backward", gout=None) == -1
    assert _call(b, _config(b), "backward", preact=None) == -1               # GELU's gradient needs z
    assert _call(b, _config(b), "backward", bias=0x700001) == -1
    assert _call(b, _config(b), "forward", bias=0x700001) == -1
    assert _call(b, _config(b), "forward", residual=b.Matrix(0x700001, 300, 1)) == -1


def test_workspace(b):
    lib = b.load()
    need = (C.c_size_t * 2)()
    query = lambda c: lib.strads_linear_workspace_bytes(c, C.cast(C.byref(need, 0), C.POINTER(C.c_size_t)), C.cast(C.byref(need, 8), C.POINTER(C.c_size_t)))
    assert query(None) == -1
    assert query(C.byref(_config(b, type=9))) == -1
    assert lib.strads_linear_workspace_bytes(C.byref(_config(b)), None, None) == -1
    c = _config(b, type=0, n_rows=1000, n_in=1000, n_out=1000)
    assert query(C.byref(c)) == 0 and need[1] > 0
    assert need[0] >= 6 * 2 * 1000 * 1000                # two operands as three bfloat16 planes
    c.x_row_stride = c.w_row_stride = 1000
    full = dict(gx=b.Matrix(0x500000, 1000, 1), gw=b.Matrix(0x600000, 1000, 1), gout=b.Matrix(0x300000, 1000, 1), preact=b.Matrix(0x400000, 1000, 1))
    c.workspace_bytes = 256
    assert _call(b, c, "backward", **full) == -3
    assert _call(b, c, "forward", out=b.Matrix(0x300000, 1000, 1)) == -3
    c.workspace, c.workspace_bytes = None, need[1]
    assert _call(b, c, "backward", **full) == -1
    # no rows: nothing to do, whatever the pointers
    c = _config(b, n_rows=0)
    c.x = None
    assert query(C.byref(c)) == 0
    assert lib.strads_linear_forward(C.byref(c), None, None, None, None) == 0
    assert lib.strads_linear_backward(C.byref(_config(b)), C.byref(b.Matrix(0x300000, 300, 1)), C.byref(b.Matrix(0x400000, 300, 1)), None, None, None) == 0
    assert lib.strads_linear_status(None) == -1


def test_the_binding_refuses(b):
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        b.linear_forward(x, torch.zeros(3, 8))           # not on a CUDA device
    with pytest.raises(ValueError):
        b.linear_forward(x[0], torch.zeros(3, 8))
