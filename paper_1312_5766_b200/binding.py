"""Thin ctypes binding of libstrads_b200.so (see include/strads.h for the contract).

Argument marshalling only: every step of the scheduled round runs in the CUDA kernels of the
library.  PyTorch is used for device memory and streams.  There is no CPU fallback: if the library
has not been built, importing its symbols raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from array import array

import torch

from . import workloads as wl

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libstrads_b200.so")

OK = 0
ERR_WORKSPACE_TOO_SMALL = -3
FLAG_UNIFORM_DRAW = 1
FLAG_NO_FILTER = 2
FLAG_SIMT_GRAM = 4
FLAG_GRAM_3XTF32 = 8
FLAG_FULL_GRAM = 16
FLAG_ABS_WEIGHT = 32
FLAG_DYNAMIC_DEPS = 64
FLAG_LOGISTIC = 128
FLAG_STALL = 256                          # sample_static only
MAX_CANDIDATES = 16384
STALL_WALK_BARRIER, STALL_GRAM_LOADS = 1, 2

EXPORTS = [
    "strads_workspace_bytes", "strads_lasso_init", "strads_round", "strads_run", "strads_round_host",
    "strads_objective", "strads_sample", "strads_filter", "strads_update", "strads_get_round",
    "strads_set_round", "strads_totals", "strads_status", "strads_colnorm2", "strads_destroy",
    "strads_error_string", "strads_last_cuda_error", "strads_profile_begin", "strads_profile_end",
    "strads_sample_static", "strads_set_wait_limit", "strads_inject_stall", "strads_recover", "strads_margin", "strads_release_cached",
    "strads_adamw_step", "strads_adamw_unpack", "strads_linear_workspace_bytes", "strads_linear_forward", "strads_linear_backward",
    "strads_linear_status",
]


class Config(C.Structure):
    _fields_ = [
        ("layout", C.c_int32),
        ("n_rows", C.c_int64), ("n_cols", C.c_int64), ("nnz", C.c_int64), ("ld", C.c_int64),
        ("x_values", C.c_void_p), ("x_row_idx", C.c_void_p), ("x_col_ptr", C.c_void_p),
        ("y", C.c_void_p), ("beta", C.c_void_p), ("resid", C.c_void_p), ("delta", C.c_void_p),
        ("lam", C.c_float), ("eta", C.c_float), ("rho", C.c_float), ("c_init", C.c_float),
        ("n_candidates", C.c_int32), ("n_keep", C.c_int32),
        ("seed", C.c_uint64),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
        ("stream", C.c_void_p),
        ("flags", C.c_uint32),
        ("n_schedulers", C.c_int32),
    ]


class RoundOut(C.Structure):
    _fields_ = [("cand", C.c_void_p), ("kept", C.c_void_p), ("dbeta", C.c_void_p), ("counts", C.c_void_p),
                ("gram", C.c_void_p)]


class AdamWTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n", C.c_int64)]


class AdamWConfig(C.Structure):
    _fields_ = [("param_type", C.c_int32), ("grad_type", C.c_int32), ("state_bits", C.c_int32),
                ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("l1", C.c_double), ("grad_scale", C.c_double), ("step", C.c_int64),
                ("lr_dev", C.c_void_p), ("grad_scale_dev", C.c_void_p), ("step_dev", C.c_void_p), ("skip_dev", C.c_void_p),
                ("stream", C.c_void_p)]


class Matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("col_stride", C.c_int64)]


class LinearConfig(C.Structure):
    _fields_ = [("type", C.c_int32), ("activation", C.c_int32), ("n_rows", C.c_int64), ("n_in", C.c_int64), ("n_out", C.c_int64),
                ("x", C.c_void_p), ("x_row_stride", C.c_int64), ("x_col_stride", C.c_int64),
                ("w", C.c_void_p), ("w_row_stride", C.c_int64), ("w_col_stride", C.c_int64), ("scale", C.c_float), ("flags", C.c_uint32), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


ACTIVATIONS = {"identity": 0, "relu": 1, "sigmoid": 2, "gelu": 3, "gelu_tanh": 4, "silu": 5}
LINEAR_FLAG_STALL = 1
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ADAMW_BLOCK = 256

_lib = None


def load() -> C.CDLL:
    """Loads the CUDA library; raises if it has not been built (no fallback of any kind)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_1312_5766_b200.build` "
                "(nvcc, sm_100a). This package has no CPU or PyTorch fallback.")
        lib = C.CDLL(LIB_PATH)
        lib.strads_error_string.restype = C.c_char_p
        lib.strads_last_cuda_error.restype = C.c_char_p
        lib.strads_workspace_bytes.argtypes = [C.POINTER(Config), C.POINTER(C.c_size_t)]
        lib.strads_lasso_init.argtypes = [C.POINTER(Config), C.POINTER(C.c_void_p)]
        lib.strads_round.argtypes = [C.c_void_p, C.POINTER(RoundOut)]
        lib.strads_run.argtypes = [C.c_void_p, C.c_int64]
        lib.strads_round_host.argtypes = [C.c_void_p] + [C.c_void_p] * 6
        lib.strads_objective.argtypes = [C.c_void_p, C.POINTER(C.c_double)]
        lib.strads_sample.argtypes = [C.c_void_p, C.c_void_p]
        lib.strads_filter.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.strads_update.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        lib.strads_get_round.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
        lib.strads_set_round.argtypes = [C.c_void_p, C.c_int64]
        lib.strads_totals.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
        lib.strads_status.argtypes = [C.c_void_p, C.POINTER(C.c_uint32)]
        lib.strads_colnorm2.argtypes = [C.c_void_p, C.POINTER(C.c_void_p)]
        lib.strads_destroy.argtypes = [C.c_void_p]
        lib.strads_profile_begin.argtypes = [C.c_void_p, C.c_int64]
        lib.strads_set_wait_limit.argtypes = [C.c_void_p, C.c_uint32]
        lib.strads_inject_stall.argtypes = [C.c_void_p, C.c_int32]
        lib.strads_recover.argtypes = [C.c_void_p]
        lib.strads_margin.argtypes = [C.c_void_p, C.POINTER(C.c_void_p)]
        lib.strads_sample_static.argtypes = [C.c_void_p, C.c_int64, C.c_float, C.c_uint64, C.c_uint64, C.c_int32,
                                             C.c_uint32, C.c_void_p, C.c_void_p]
        lib.strads_linear_workspace_bytes.argtypes = [C.POINTER(LinearConfig), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        lib.strads_linear_forward.argtypes = [C.POINTER(LinearConfig), C.c_void_p] + [C.POINTER(Matrix)] * 3
        lib.strads_linear_backward.argtypes = [C.POINTER(LinearConfig)] + [C.POINTER(Matrix)] * 4 + [C.c_void_p]
        lib.strads_linear_status.argtypes = [C.POINTER(C.c_uint32)]
        lib.strads_adamw_step.argtypes = [C.POINTER(AdamWConfig), C.POINTER(AdamWTensor), C.c_int32]
        lib.strads_adamw_unpack.argtypes = [C.POINTER(AdamWTensor), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_int32,
                                            C.c_void_p]
        lib.strads_profile_end.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        _lib = lib
    return _lib


class StradsError(RuntimeError):
    def __init__(self, code: int, where: str):
        lib = load()
        msg = lib.strads_error_string(code).decode()
        cuda = lib.strads_last_cuda_error().decode()
        super().__init__(f"{where}: {msg} ({code})" + (f" [{cuda}]" if code == -4 and cuda else ""))
        self.code = code


def _check(code: int, where: str) -> None:
    if code != OK:
        raise StradsError(code, where)


def _ptr(t: torch.Tensor | None):
    return None if t is None else C.c_void_p(t.data_ptr())


def workspace_bytes(layout, n_rows, n_cols, n_candidates, n_keep, nnz=0, ld=None) -> int:
    cfg = Config()
    cfg.layout, cfg.n_rows, cfg.n_cols, cfg.nnz = layout, n_rows, n_cols, nnz
    cfg.ld = ld if ld is not None else (n_rows + 3) // 4 * 4
    cfg.n_candidates, cfg.n_keep = n_candidates, n_keep
    out = C.c_size_t(0)
    _check(load().strads_workspace_bytes(C.byref(cfg), C.byref(out)), "strads_workspace_bytes")
    return int(out.value)


STATIC_MAX_CANDIDATES = 4096


def sample_static(delta: torch.Tensor, eta: float, seed: int, t: int, n_candidates: int, flags: int = 0,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """Candidate draw without a handle or workspace (strads_sample_static): for callers that cannot
    allocate device memory.  `out` (int32 [n_candidates], device) is allocated here only if not given."""
    assert delta.is_cuda and delta.dtype == torch.float32 and delta.is_contiguous()
    if out is None:
        out = torch.empty(n_candidates, dtype=torch.int32, device=delta.device)
    with torch.cuda.device(delta.device):
        stream = torch.cuda.current_stream().cuda_stream
        _check(load().strads_sample_static(_ptr(delta), int(delta.numel()), float(eta), int(seed), int(t),
                                           int(n_candidates), int(flags), _ptr(out), C.c_void_p(stream)),
               "strads_sample_static")
    return out


class StradsLasso:
    """One Lasso problem resident on a CUDA device, stepped by the library's kernels.

    x_values / row_idx / col_ptr / y are torch CUDA tensors owned by the caller (kept alive here);
    beta, resid, delta and the workspace are allocated here as torch tensors.
    """

    def __init__(self, layout, n_rows, n_cols, values, y, lam, eta, rho, n_candidates, n_keep, seed=0,
                 row_idx=None, col_ptr=None, c_init=1e4, flags=0, beta0=None, stream=None, n_schedulers=1):
        lib = load()
        dev = values.device
        assert dev.type == "cuda", "the design matrix must live on a CUDA device"
        self.layout, self.N, self.J = int(layout), int(n_rows), int(n_cols)
        self.n_candidates, self.n_keep = int(n_candidates), int(n_keep)
        self.values, self.row_idx, self.col_ptr, self.y = values, row_idx, col_ptr, y
        self.lam, self.eta, self.rho = float(lam), float(eta), float(rho)
        assert values.dtype == torch.float32 and y.dtype == torch.float32 and values.is_contiguous()
        ld = int(values.shape[1]) if layout == wl.DENSE else 0
        nnz = int(values.numel()) if layout == wl.CSC else 0
        if layout == wl.CSC:
            assert row_idx.dtype == torch.int32 and col_ptr.dtype == torch.int64
        self.beta = torch.zeros(self.J, dtype=torch.float32, device=dev) if beta0 is None else \
            beta0.to(device=dev, dtype=torch.float32).contiguous().clone()
        self.resid = torch.empty(self.N, dtype=torch.float32, device=dev)
        self.delta = torch.empty(self.J, dtype=torch.float32, device=dev)
        self.stream = stream
        cfg = Config()
        cfg.layout, cfg.n_rows, cfg.n_cols, cfg.nnz, cfg.ld = self.layout, self.N, self.J, nnz, ld
        cfg.n_candidates, cfg.n_keep = self.n_candidates, self.n_keep
        self.n_schedulers = cfg.n_schedulers = int(n_schedulers)
        cfg.flags = flags                      # (the logistic loss adds the margin to the workspace; rho left open: buffers for rounds in one launch)
        need = C.c_size_t(0)
        _check(lib.strads_workspace_bytes(C.byref(cfg), C.byref(need)), "strads_workspace_bytes")
        self.workspace = torch.empty(int(need.value), dtype=torch.uint8, device=dev)
        cfg.x_values, cfg.x_row_idx, cfg.x_col_ptr = values.data_ptr(), \
            (row_idx.data_ptr() if row_idx is not None else None), (col_ptr.data_ptr() if col_ptr is not None else None)
        cfg.y, cfg.beta, cfg.resid, cfg.delta = y.data_ptr(), self.beta.data_ptr(), self.resid.data_ptr(), \
            self.delta.data_ptr()
        cfg.lam, cfg.eta, cfg.rho, cfg.c_init = lam, eta, rho, c_init
        cfg.seed = seed
        cfg.workspace, cfg.workspace_bytes = self.workspace.data_ptr(), int(need.value)
        cfg.stream = None if stream is None else stream.cuda_stream
        cfg.flags = flags
        self._cfg = cfg
        self._h = C.c_void_p(None)
        with torch.cuda.device(dev):
            _check(lib.strads_lasso_init(C.byref(cfg), C.byref(self._h)), "strads_lasso_init")
        self._dev = dev
        # per-round output buffers (device)
        self.cand = torch.empty(self.n_candidates, dtype=torch.int32, device=dev)
        self.kept = torch.empty(self.n_keep, dtype=torch.int32, device=dev)
        self.dbeta = torch.empty(self.n_keep, dtype=torch.float32, device=dev)
        self.counts = torch.zeros(4, dtype=torch.int32, device=dev)

    @classmethod
    def from_problem(cls, p: wl.LassoProblem, device="cuda", **kw):
        mv = lambda t: None if t is None else t.to(device)
        return cls(p.layout, p.n_rows, p.n_cols, mv(p.values), mv(p.y), p.lam, p.eta, p.rho, p.n_candidates,
                   p.n_keep, seed=p.seed, row_idx=mv(p.row_idx), col_ptr=mv(p.col_ptr), **kw)

    # ---- whole rounds ----
    def round(self, want_gram: bool = False):
        """One round; returns (cand, kept, dbeta, counts) device tensors (reused between calls)."""
        out = RoundOut(self.cand.data_ptr(), self.kept.data_ptr(), self.dbeta.data_ptr(), self.counts.data_ptr(), None)
        gram = None
        if want_gram:
            gram = torch.zeros((self.n_candidates, self.n_candidates), dtype=torch.float32, device=self._dev)
            out.gram = gram.data_ptr()
        _check(load().strads_round(self._h, C.byref(out)), "strads_round")
        return (self.cand, self.kept, self.dbeta, self.counts) + ((gram,) if want_gram else ())

    def run(self, n_rounds: int) -> None:
        _check(load().strads_run(self._h, int(n_rounds)), "strads_run")

    def round_host(self, beta_h, resid_h, delta_h, kept_h=None, dbeta_h=None, counts_h=None) -> None:
        """One round on state held in (pinned) host tensors; see strads_round_host."""
        _check(load().strads_round_host(self._h, _ptr(beta_h), _ptr(resid_h), _ptr(delta_h), _ptr(kept_h),
                                        _ptr(dbeta_h), _ptr(counts_h)), "strads_round_host")

    def objective(self) -> float:
        out = C.c_double(0.0)
        _check(load().strads_objective(self._h, C.byref(out)), "strads_objective")
        return float(out.value)

    # ---- split-phase ----
    def sample(self) -> torch.Tensor:
        _check(load().strads_sample(self._h, _ptr(self.cand)), "strads_sample")
        return self.cand

    def filter(self, cand: torch.Tensor, want_gram: bool = False):
        n = int(cand.numel())
        gram = torch.zeros((n, n), dtype=torch.float32, device=self._dev) if want_gram else None
        _check(load().strads_filter(self._h, _ptr(cand), n, _ptr(self.kept), _ptr(self.counts), _ptr(gram)),
               "strads_filter")
        return (self.kept, self.counts) + ((gram,) if want_gram else ())

    def update(self, kept: torch.Tensor) -> torch.Tensor:
        _check(load().strads_update(self._h, _ptr(kept), int(kept.numel()), _ptr(self.dbeta)), "strads_update")
        return self.dbeta

    # ---- bookkeeping ----
    def get_round(self) -> int:
        t = C.c_int64(0)
        _check(load().strads_get_round(self._h, C.byref(t)), "strads_get_round")
        return int(t.value)

    def set_round(self, t: int) -> None:
        _check(load().strads_set_round(self._h, int(t)), "strads_set_round")

    def totals(self) -> dict:
        t = (C.c_int64 * 4)()
        _check(load().strads_totals(self._h, t), "strads_totals")
        return {"rounds": t[0], "examined": t[1], "kept": t[2], "nonzero": t[3]}

    def status(self) -> tuple[int, int]:
        bits = C.c_uint32(0)
        rc = load().strads_status(self._h, C.byref(bits))
        return rc, int(bits.value)

    def set_wait_limit(self, iterations: int) -> None:
        _check(load().strads_set_wait_limit(self._h, int(iterations)), "strads_set_wait_limit")

    def inject_stall(self, which: int) -> None:
        _check(load().strads_inject_stall(self._h, int(which)), "strads_inject_stall")

    def recover(self) -> None:
        _check(load().strads_recover(self._h), "strads_recover")

    def colnorm2(self) -> torch.Tensor:
        """||x_j||^2 (FP64), a view into the workspace."""
        ptr = C.c_void_p(None)
        _check(load().strads_colnorm2(self._h, C.byref(ptr)), "strads_colnorm2")
        off = ptr.value - self.workspace.data_ptr()
        return self.workspace[off:off + 8 * self.J].view(torch.float64)

    def margin(self) -> torch.Tensor:
        """The margin X beta (FP32), a view into the workspace (logistic loss only)."""
        ptr = C.c_void_p(None)
        _check(load().strads_margin(self._h, C.byref(ptr)), "strads_margin")
        off = ptr.value - self.workspace.data_ptr()
        return self.workspace[off:off + 4 * self.N].view(torch.float32)

    def profile_begin(self, max_rounds: int) -> None:
        _check(load().strads_profile_begin(self._h, int(max_rounds)), "strads_profile_begin")

    def profile_end(self) -> dict:
        ms = (C.c_double * 5)()
        n = C.c_int64(0)
        _check(load().strads_profile_end(self._h, ms, C.byref(n)), "strads_profile_end")
        return {"rounds": int(n.value), "sample_ms": ms[0], "pack_ms": ms[1], "gram_ms": ms[2], "walk_ms": ms[3],
                "update_ms": ms[4]}

    def close(self) -> None:
        if self._h:
            load().strads_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _refuse(t, what, dtype, index, shape):
    if t.dtype != dtype:
        raise TypeError(f"{what} of type {t.dtype}, {dtype} expected")
    if t.get_device() != index:
        raise ValueError(f"{what} on {t.device}, cuda:{index} expected")
    raise ValueError(f"{what} must be {'contiguous, ' if len(shape) == 1 else ''}of shape {tuple(shape)}, not {tuple(t.shape)}")


def _matrix(t, what, dtype, index, shape):
    """A tensor as the library takes it; refuses other types, devices and shapes than those of the call."""
    if t.dtype != dtype or t.get_device() != index or t.shape != shape:
        _refuse(t, what, dtype, index, shape)
    rs, cs = t.stride()
    return Matrix(t.data_ptr(), rs, cs)


def _vector(t, what, dtype, index, n):
    if t.dtype != dtype or t.get_device() != index or t.shape != (n,) or not t.is_contiguous():
        _refuse(t, what, dtype, index, (n,))
    return t.data_ptr()


def _refuse_autograd(where):
    """The layers record nothing: a result that quietly had no gradient would be lost to the program that asks for one."""
    raise RuntimeError(f"{where} records nothing for autograd: call it under torch.no_grad(), or with detached tensors, and linear_backward for the gradient")


def _linear_config(x, w, activation, scale, flags):
    xs, ws = x.shape, w.shape
    if len(xs) != 2 or len(ws) != 2:
        raise ValueError("x and w must have two dimensions")
    index, dtype = x.get_device(), x.dtype
    if index < 0:
        raise ValueError("x must live on a CUDA device")
    if dtype not in TYPES:
        raise TypeError(f"x of type {dtype}")
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation {activation!r}: one of {', '.join(ACTIVATIONS)}")
    n, k = xs
    m = ws[0]
    if w.dtype != dtype or w.get_device() != index or ws[1] != k:
        _refuse(w, "w", dtype, index, (m, k))
    xr, xc = x.stride()
    wr, wc = w.stride()
    cfg = LinearConfig(TYPES[dtype], ACTIVATIONS[activation], n, k, m, x.data_ptr(), xr, xc, w.data_ptr(), wr, wc, scale, flags, None, 0,
                       torch._C._cuda_getCurrentRawStream(index))
    return cfg, n, k, m, dtype, index


def _linear_call(call, where, cfg, which, device):
    """The call with no workspace, and where it needs one with one from the caching allocator, on the current stream, so that two
    calls only share one where they follow each other."""
    rc = call()
    if rc == ERR_WORKSPACE_TOO_SMALL:
        need = (C.c_size_t(0), C.c_size_t(0))
        _check(load().strads_linear_workspace_bytes(C.byref(cfg), C.byref(need[0]), C.byref(need[1])), "strads_linear_workspace_bytes")
        ws = torch.empty(need[which].value, dtype=torch.uint8, device=device)
        cfg.workspace, cfg.workspace_bytes = ws.data_ptr(), need[which].value
        rc = call()
    if rc != OK:
        _check(rc, where)


def linear_forward(x, w, bias=None, residual=None, activation="identity", scale=1.0, want_preact=False, out=None, preact=None, flags=0):
    """out = residual + scale * activation(x w^T + bias) (strads_linear_forward).  x [n_rows, n_in] and w [n_out, n_in] in either
    order, float32, bfloat16 or float16; residual [n_rows, n_out] may be an expanded tensor, and out may be the residual itself.
    Returns out, and with want_preact (or preact, a tensor for it) the pair (out, x w^T + bias).  Nothing is recorded for autograd (linear_backward is the
    gradient): while that is on, tensors that require a gradient are refused."""
    if torch.is_grad_enabled() and (x.requires_grad or w.requires_grad or (bias is not None and bias.requires_grad) or
                                    (residual is not None and residual.requires_grad) or (out is not None and out.requires_grad) or
                                    (preact is not None and preact.requires_grad)):
        _refuse_autograd("linear_forward")
    cfg, n, _, m, dtype, index = _linear_config(x, w, activation, scale, flags)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return linear_forward(x, w, bias, residual, activation, scale, want_preact, out, preact, flags)
    lib, shape = load(), (n, m)
    b = None if bias is None else _vector(bias, "bias", dtype, index, m)
    r = None if residual is None else C.byref(_matrix(residual, "residual", dtype, index, shape))
    if out is None:
        out = x.new_empty(shape)
    if preact is None and want_preact:
        preact = x.new_empty(shape)
    o = C.byref(_matrix(out, "out", dtype, index, shape))
    z = None if preact is None else C.byref(_matrix(preact, "preact", dtype, index, shape))
    _linear_call(lambda: lib.strads_linear_forward(C.byref(cfg), b, r, o, z), "strads_linear_forward", cfg, 0, x.device)
    return out if preact is None else (out, preact)


def _empty_in_order_of(t):
    return t.new_empty(t.shape[::-1]).t() if t.stride(0) < t.stride(1) else t.new_empty(t.shape)


def linear_backward(grad_out, x, w, preact=None, activation="identity", scale=1.0, want_x=True, want_w=True, want_bias=True,
                    grad_x=None, grad_w=None, grad_bias=None, flags=0):
    """Gradients of linear_forward (strads_linear_backward) from grad_out [n_rows, n_out] and the preact that the forward pass gave
    (not with the identity): (grad_x, grad_w, grad_bias), None where not wanted.  New gradients have the order of x and w.  The residual's
    gradient is grad_out itself.  Not differentiable itself: as in linear_forward, tensors that require a gradient are refused while autograd is on."""
    if torch.is_grad_enabled() and (grad_out.requires_grad or x.requires_grad or w.requires_grad or (preact is not None and preact.requires_grad) or
                                    (grad_x is not None and grad_x.requires_grad) or (grad_w is not None and grad_w.requires_grad) or
                                    (grad_bias is not None and grad_bias.requires_grad)):
        _refuse_autograd("linear_backward")
    cfg, n, k, m, dtype, index = _linear_config(x, w, activation, scale, flags)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return linear_backward(grad_out, x, w, preact, activation, scale, want_x, want_w, want_bias, grad_x, grad_w, grad_bias, flags)
    lib, shape = load(), (n, m)
    g = C.byref(_matrix(grad_out, "grad_out", dtype, index, shape))
    if preact is None and activation != "identity":
        raise ValueError("the gradient needs preact")
    z = None if preact is None else C.byref(_matrix(preact, "preact", dtype, index, shape))
    if want_x and grad_x is None:
        grad_x = _empty_in_order_of(x)
    if want_w and grad_w is None:
        grad_w = _empty_in_order_of(w)
    if want_bias and grad_bias is None:
        grad_bias = x.new_empty(m)
    gx = None if grad_x is None else C.byref(_matrix(grad_x, "grad_x", dtype, index, (n, k)))
    gw = None if grad_w is None else C.byref(_matrix(grad_w, "grad_w", dtype, index, (m, k)))
    gb = None if grad_bias is None else _vector(grad_bias, "grad_bias", dtype, index, m)
    _linear_call(lambda: lib.strads_linear_backward(C.byref(cfg), g, z, gx, gw, gb), "strads_linear_backward", cfg, 1, x.device)
    return grad_x, grad_w, grad_bias


def linear_status(device=None) -> tuple[int, int]:
    """(code, bits) of the linear layers' bounded waits on a device since the last call of this (waits for the device)."""
    bits = C.c_uint32(0)
    with torch.cuda.device(device):
        rc = load().strads_linear_status(C.byref(bits))
    return rc, int(bits.value)


class AdamW:
    """AdamW over many tensors at once, moments in 32 or in 8 bits (strads_adamw_step).

    params are contiguous tensors of one type (float32, bfloat16, float16) on one CUDA device, stepped in place; masters,
    with 16-bit parameters, their float32 copies, which then take the step.  Where their storage is replaced (p.data = .., set_, a
    module's .to()) the next step goes where they are then, or refuses what no longer fits.  moments, where given, are used as they are and
    kept up to date: (first, second), lists of float32 tensors, with bits=32; (codes, scales, codes, scales), lists of
    int8, float32, uint8 and float32 tensors, with bits=8 (a scale per block of 256 elements).  Otherwise they are allocated
    here, as noughts, in the parameters' shapes.  Either way their memory is this object's from then on: `state` and `moments` give views of
    it, and a given tensor whose storage is replaced later is no longer one.
    """

    def __init__(self, params, bits=32, masters=None, moments=None, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, l1=0.0):
        params = list(params)
        if bits not in (32, 8):
            raise ValueError("bits must be 32 or 8")
        if not params:
            raise ValueError("no parameters")
        dtype, dev = params[0].dtype, params[0].device
        if dtype not in TYPES:
            raise TypeError(f"parameters of type {dtype}")
        if dev.type != "cuda":
            raise ValueError("the parameters must live on a CUDA device")
        if masters is not None and dtype == torch.float32:
            raise ValueError("masters go with 16-bit parameters")
        self.params, self.bits, self.device, self.dtype = params, bits, dev, dtype
        self.masters = None if masters is None else list(masters)
        sizes = [p.numel() for p in params]
        blocks = [-(-n // ADAMW_BLOCK) for n in sizes]
        if bits == 32:
            kinds = [(torch.float32, sizes)] * 2
        else:
            kinds = [(torch.int8, sizes), (torch.float32, blocks), (torch.uint8, sizes), (torch.float32, blocks)]
        if moments is None:
            moments = [self._noughts(t, [p.shape for p in params] if n is sizes else [(k,) for k in n], dev) for t, n in kinds]
        self._state = [[t.detach() for t in m] for m in moments]      # views that nobody else can give another storage
        if len(self._state) != len(kinds):
            raise ValueError(f"{len(kinds)} lists of moments expected with {bits} bits")
        self._kinds, self._sizes, self._index = kinds, sizes, dev.index
        self._cfg = AdamWConfig(param_type=TYPES[dtype], state_bits=bits, beta1=betas[0], beta2=betas[1], eps=eps,
                                weight_decay=weight_decay, l1=l1)
        self._list = (AdamWTensor * len(params))()
        words = memoryview(self._list).cast("B").cast("Q")
        self._grads = words[AdamWTensor.grad.offset // 8::C.sizeof(AdamWTensor) // 8]
        self._bind()

    def _addresses(self):
        """Where parameters and masters are now."""
        at = list(map(torch.Tensor.data_ptr, self.params))
        return at if self.masters is None else at + list(map(torch.Tensor.data_ptr, self.masters))

    def _bind(self):
        """Takes the tensors as they are now into the list that a step passes on, if they fit."""
        self._at = None
        self._check("parameters", self.params, self.dtype, self._sizes)
        if self.masters is not None:
            self._check("masters", self.masters, torch.float32, self._sizes)
        for m, (t, n) in zip(self._state, self._kinds):
            self._check("moments", m, t, n)
        written = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())
                         for group in (self.params, self.masters or [], *self._state) for t in group if t.numel())
        if any(a[1] > b[0] for a, b in zip(written, written[1:])):
            raise ValueError("parameters, masters and moments must not share memory")
        for i, p in enumerate(self.params):
            e = self._list[i]
            e.param, e.n = p.data_ptr(), p.numel()
            e.master = self.masters[i].data_ptr() if self.masters is not None else None
            e.m, e.v = self._state[0][i].data_ptr(), self._state[1 if self.bits == 32 else 2][i].data_ptr()
            if self.bits == 8:
                e.m_scale, e.v_scale = self._state[1][i].data_ptr(), self._state[3][i].data_ptr()
        self._at = self._addresses()

    @property
    def state(self):
        """The moments as they are held: (first, second), or (codes, scales, codes, scales) of both with bits=8, lists of views."""
        return [[t.detach() for t in m] for m in self._state]

    @staticmethod
    def _noughts(dtype, shapes, dev):
        starts, total = [], 0
        for s in shapes:                                 # every tensor's part starts on 16 bytes
            starts.append(total)
            total += -(-math.prod(s) // 16) * 16
        flat = torch.zeros(total, dtype=dtype, device=dev)
        return [flat[a:a + math.prod(s)].view(s) for a, s in zip(starts, shapes)]

    def _check(self, what, tensors, dtype, sizes):
        if len(tensors) != len(sizes):
            raise ValueError(f"{len(tensors)} {what} for {len(sizes)} parameters")
        for t, n in zip(tensors, sizes):
            if t.device != self.device or not t.is_contiguous() or t.numel() != n:
                raise ValueError(f"{what} must be contiguous, of the parameters' sizes and on their device")
            if t.dtype != dtype:
                raise TypeError(f"{what} of type {t.dtype}, {dtype} expected")

    def _value(self, v, dtype, default):
        """A number, or the default and the address of one on the device."""
        if type(v) is float or type(v) is int or not isinstance(v, torch.Tensor):      # (asking a number whether it is a tensor takes longer)
            return v, None
        return default, self._scalar(v, dtype)

    def _scalar(self, t, dtype):
        if t.device != self.device or t.dtype != dtype or t.numel() != 1:
            raise ValueError(f"a scalar on the device must be one {dtype} on {self.device}")
        return t.data_ptr()

    def step(self, grads, lr=1e-3, step=1, grad_scale=1.0, skip=None):
        """One step with the given gradients (float32 or the parameters' type, contiguous).  `step` counts from 1.  lr (float32),
        step (int64), grad_scale (float32) and skip (int32) may be one-element tensors on the device, read when the
        step runs: a captured step then follows them; skip other than 0 leaves everything as it is."""
        grads = list(grads)
        gtype = grads[0].dtype if grads else None
        if gtype is not torch.float32 and gtype is not self.dtype:
            raise TypeError(f"gradients of type {gtype}")
        if (list(map(torch.Tensor.numel, grads)) != self._sizes or {g.dtype for g in grads} != {gtype} or
                set(map(torch.Tensor.get_device, grads)) != {self._index} or not all(map(torch.Tensor.is_contiguous, grads))):
            self._check("gradients", grads, gtype, self._sizes)
        if self._addresses() != self._at:
            self._bind()
        if self._index != torch._C._cuda_getDevice():
            with torch.cuda.device(self._index):
                return self.step(grads, lr, step, grad_scale, skip)
        c = self._cfg
        c.grad_type = TYPES[gtype]
        c.lr, c.lr_dev = self._value(lr, torch.float32, 0.0)
        c.step, c.step_dev = self._value(step, torch.int64, 1)
        c.grad_scale, c.grad_scale_dev = self._value(grad_scale, torch.float32, 1.0)
        c.skip_dev = None if skip is None else self._scalar(skip, torch.int32)
        self._grads[:] = array("Q", map(torch.Tensor.data_ptr, grads))
        c.stream = torch._C._cuda_getCurrentRawStream(self._index)
        rc = load().strads_adamw_step(C.byref(c), self._list, len(grads))
        if rc != OK:
            _check(rc, "strads_adamw_step")

    def moments(self, out=None):
        """(first, second): the moments as lists of float32 tensors.  32 bits: the state itself.  8 bits: the values that the
        codes stand for, in new tensors or in `out`, a pair of lists of contiguous float32 tensors."""
        if self.bits == 32:
            return tuple(self.state)
        sizes = [p.numel() for p in self.params]
        if out is None:
            out = [self._noughts(torch.float32, [p.shape for p in self.params], self.device) for _ in range(2)]
        first, second = (list(t) for t in out)
        self._check("values", first, torch.float32, sizes)
        self._check("values", second, torch.float32, sizes)
        n = len(sizes)
        ptrs = [(C.c_void_p * n)(*[t.data_ptr() or None for t in group]) for group in (first, second)]
        with torch.cuda.device(self.device):
            _check(load().strads_adamw_unpack(self._list, *ptrs, n, C.c_void_p(torch.cuda.current_stream().cuda_stream)),
                   "strads_adamw_unpack")
        return first, second
