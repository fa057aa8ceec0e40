"""Thin ctypes binding over libfd.so: same names as include/fd.h, argument marshalling only.

PyTorch is used for device memory and streams, nothing else: every step of the path runs in
the library's own CUDA kernels.  There is no CPU fallback; if the library cannot be loaded the
import fails loudly.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from ctypes import POINTER, Structure, byref, c_char_p, c_double, c_int32, c_int64, c_size_t, c_void_p

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfd.so")

FD_OK, FD_ERR_INVALID, FD_ERR_WORKSPACE, FD_ERR_CUDA, FD_ERR_NOT_CONVERGED = 0, 1, 2, 3, 4
FD_ERR_PERRON_WALL, FD_ERR_UNSUPPORTED, FD_ERR_TIMEOUT, FD_ERR_NONFINITE, FD_ERR_COMM = 5, 6, 7, 8, 9
FD_PREC_FP32, FD_PREC_FAST = 0, 1
FD_PATH_AUTO, FD_PATH_SIMT, FD_PATH_TC = 0, 1, 2
FD_FLOW_VERTEX, FD_FLOW_PERRON_WALL, FD_FLOW_LEFT_EDGE, FD_FLOW_RIGHT_EDGE = 0, 1, 2, 3
FD_BF16, FD_FP16, FD_FP32 = 0, 1, 2
FD_ROTARY_HALF, FD_ROTARY_INTERLEAVED = 0, 1
FD_ROTARY_PLAIN, FD_ROTARY_LINEAR, FD_ROTARY_BASE, FD_ROTARY_RAMP = 0, 1, 2, 3
FLOW_OUTCOMES = {0: "VERTEX", 1: "PERRON_WALL", 2: "LEFT_EDGE", 3: "RIGHT_EDGE"}

# Every symbol include/fd.h declares (checked by the CPU test-suite against the header).
EXPORTS = [
    "fd_workspace_bytes", "fd_create", "fd_destroy", "fd_set_option", "fd_get_option", "fd_beta0", "fd_degree",
    "fd_apply", "fd_apply_general", "fd_synchronize", "fd_eigs", "fd_beta_flow", "fd_beta_flow_cascade", "fd_nystrom", "fd_ladder_start", "fd_scale_by_degree",
    "fd_apply_general_static", "fd_unit_peaks", "fd_shard_rows", "fd_shard_exchange_bytes", "fd_set_shard", "fd_rotary_frequencies", "fd_rotary",
    "fd_kv_create", "fd_kv_destroy", "fd_kv_synchronize", "fd_kv_append", "fd_kv_attend_bytes", "fd_kv_attend", "fd_kv_evict", "fd_status_string", "fd_last_error", "fd_version", "fd_launch_count",
]


class fd_eigs_info(Structure):
    _fields_ = [("applies", c_int32), ("restarts", c_int32), ("converged", c_int32), ("basis_cols", c_int32),
                ("max_residual", c_double), ("seconds_apply", c_double), ("seconds_total", c_double)]


class fd_unit_rates(Structure):
    _fields_ = [("sm_count", c_int32)] + [(n, c_double) for n in (
        "ex2_per_clk_sm", "ffma_per_clk_sm", "cvt_f16x2_per_clk_sm", "lop_per_clk_sm", "fadd_per_clk_sm",
        "clk_mma_ts_n64", "clk_mma_ts_n128", "clk_mma_ss_n64", "clk_mma_ss_n128")]


class fd_probe(Structure):
    _fields_ = [(n, c_double) for n in ("beta", "S_off", "S_off_2beta", "n_eff", "d_hat", "V_bias", "V_stat", "V_mach",
                                        "V", "g_P", "lambda1")] + [("applies", c_int32), ("flags", c_int32)]


class fd_flow_opts(Structure):
    _fields_ = [("beta_start", c_double), ("beta_max", c_double), ("ratio", c_double), ("alpha", c_double),
                ("eta", c_double), ("tol", c_double), ("k", c_int32), ("b", c_int32), ("max_applies", c_int32),
                ("warm_start", c_int32)]


class fd_cascade_stage(Structure):
    _fields_ = [("prec", c_int32), ("eta", c_double), ("tol", c_double)]


class fd_heads(Structure):
    _fields_ = [("p_dev", c_void_p), ("token_stride", c_int64), ("head_stride", c_int64), ("heads", c_int32)]


class fd_kv_desc(Structure):
    _fields_ = ([("k_dev", c_void_p), ("v_dev", c_void_p)] + [(n, c_int64) for n in (
        "k_page_stride", "k_token_stride", "k_head_stride", "v_page_stride", "v_token_stride", "v_head_stride")]
        + [(n, c_int32) for n in ("num_pages", "page_size", "heads", "head_dim", "dtype")] + [("status_dev", c_void_p)])


class fd_kv_batch(Structure):
    _fields_ = [("table_dev", c_void_p), ("table_stride", c_int64), ("kv_len_dev", c_void_p), ("q_start_dev", c_void_p)] + [
        (n, c_int32) for n in ("batch", "max_pages", "total_q", "max_new", "max_len")]


class fd_kv_append_args(Structure):
    _fields_ = [("k", fd_heads), ("v", fd_heads), ("q", fd_heads), ("q_out", fd_heads), ("positions_dev", c_void_p),
                ("freqs_dev", c_void_p), ("scale", c_double), ("rot_dim", c_int32), ("layout", c_int32)]


class fd_kv_attend_args(Structure):
    _fields_ = [("q", fd_heads), ("out", fd_heads), ("scale", c_double), ("causal", c_int32), ("window", c_int32),
                ("lse_dev", c_void_p), ("weights_in_dev", c_void_p), ("weights_out_dev", c_void_p), ("weights_stride", c_int64)]


class fd_kv_evict_args(Structure):
    _fields_ = [("weights_in_dev", c_void_p), ("weights_out_dev", c_void_p), ("weights_stride", c_int64),
                ("new_table_dev", c_void_p), ("new_table_stride", c_int64), ("new_max_pages", c_int32), ("keep", c_int32),
                ("first", c_int32), ("recent", c_int32), ("kept_dev", c_void_p), ("new_len_dev", c_void_p)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(the CUDA library is the product; there is no fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    lib.fd_workspace_bytes.argtypes = [c_int64, c_int32, c_int32, c_int32]
    lib.fd_workspace_bytes.restype = c_size_t
    lib.fd_create.argtypes = [POINTER(c_void_p), c_void_p, c_int64, c_int32, c_int64, c_int32, c_int32, c_int32,
                              c_void_p, c_size_t, c_void_p]
    lib.fd_destroy.argtypes = [c_void_p]
    lib.fd_set_option.argtypes = [c_void_p, c_char_p, c_double]
    lib.fd_get_option.argtypes = [c_void_p, c_char_p, POINTER(c_double)]
    lib.fd_beta0.argtypes = [c_void_p, POINTER(c_double)]
    lib.fd_degree.argtypes = [c_void_p, c_double, c_double, c_int32, c_void_p, c_void_p, c_void_p,
                              POINTER(c_double), POINTER(c_double)]
    lib.fd_synchronize.argtypes = [c_void_p]
    lib.fd_apply.argtypes = [c_void_p, c_void_p, c_int64, c_int32, c_void_p, c_int64, c_int32]
    lib.fd_apply_general.argtypes = [c_void_p, c_double, c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_void_p,
                                     c_int64, c_int32, c_void_p, c_int64, c_int32]
    lib.fd_eigs.argtypes = [c_void_p, c_int32, c_int32, c_double, c_int32, c_void_p, c_int64, c_int32,
                            POINTER(c_double), c_void_p, c_int64, POINTER(fd_eigs_info)]
    lib.fd_beta_flow.argtypes = [c_void_p, POINTER(fd_flow_opts), c_void_p, c_int64, c_int32, POINTER(fd_probe),
                                 POINTER(c_int32), POINTER(c_int32), POINTER(c_double), POINTER(c_double), c_void_p,
                                 c_int64]
    lib.fd_beta_flow_cascade.argtypes = [c_void_p, POINTER(fd_flow_opts), POINTER(fd_cascade_stage), c_int32, c_void_p,
                                         c_int64, c_int32, POINTER(fd_probe), POINTER(c_int32), POINTER(c_int32),
                                         POINTER(c_int32), POINTER(c_double), POINTER(c_double), c_void_p, c_int64]
    lib.fd_nystrom.argtypes = [c_void_p, c_void_p, c_int64, c_int64, c_void_p, c_int64, c_int32, POINTER(c_double),
                               c_void_p, c_int64]
    lib.fd_ladder_start.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_int32, POINTER(c_double),
                                    c_void_p, c_int64]
    lib.fd_ladder_start.restype = c_int32
    lib.fd_scale_by_degree.argtypes = [c_void_p, c_void_p, c_int64, c_int32, c_double, c_void_p, c_int64]
    for name in ("fd_synchronize", "fd_create", "fd_destroy", "fd_set_option", "fd_get_option", "fd_beta0", "fd_degree", "fd_apply",
                 "fd_apply_general", "fd_eigs", "fd_beta_flow", "fd_beta_flow_cascade", "fd_nystrom", "fd_scale_by_degree"):
        getattr(lib, name).restype = c_int32
    lib.fd_apply_general_static.argtypes = [c_void_p, c_int64, c_int32, c_int64, c_double, c_void_p, c_void_p, c_void_p,
                                            c_int64, c_int32, c_void_p, c_int64, c_void_p, ctypes.c_char_p, c_size_t]
    lib.fd_apply_general_static.restype = c_int32
    lib.fd_unit_peaks.argtypes = [c_void_p, c_size_t, c_void_p, POINTER(fd_unit_rates)]
    lib.fd_unit_peaks.restype = c_int32
    lib.fd_rotary_frequencies.argtypes = [c_int32, c_double, c_int32, c_double, c_double, c_double, c_double, POINTER(c_double)]
    # (structures of arguments come as pointers or as packed bytes: see _HEADS)
    lib.fd_rotary.argtypes = [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p, c_int32, c_int32,
                              c_double, c_int32, c_void_p, c_char_p, c_size_t]
    lib.fd_kv_create.argtypes = [POINTER(c_void_p), POINTER(fd_kv_desc), c_char_p, c_size_t]
    lib.fd_kv_destroy.argtypes = [c_void_p]
    lib.fd_kv_destroy.restype = None
    lib.fd_kv_synchronize.argtypes = [c_void_p, c_void_p]
    lib.fd_kv_append.argtypes = [c_void_p, POINTER(fd_kv_batch), c_void_p, c_void_p, c_char_p, c_size_t]
    lib.fd_kv_attend_bytes.argtypes = [c_void_p, POINTER(fd_kv_batch), c_int32, c_int32]
    lib.fd_kv_attend_bytes.restype = c_size_t
    lib.fd_kv_attend.argtypes = [c_void_p, POINTER(fd_kv_batch), c_void_p, c_void_p, c_size_t, c_void_p, c_char_p, c_size_t]
    lib.fd_kv_evict.argtypes = [c_void_p, POINTER(fd_kv_batch), c_void_p, c_void_p, c_char_p, c_size_t]
    for name in ("fd_rotary_frequencies", "fd_rotary", "fd_kv_create", "fd_kv_synchronize", "fd_kv_append", "fd_kv_attend", "fd_kv_evict"):
        getattr(lib, name).restype = c_int32
    lib.fd_status_string.argtypes = [c_int32]
    lib.fd_status_string.restype = c_char_p
    lib.fd_last_error.argtypes = [c_void_p]
    lib.fd_last_error.restype = c_char_p
    lib.fd_version.restype = c_int32
    lib.fd_launch_count.restype = c_int64
    return lib


lib = _load()


class FdError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        msg = lib.fd_status_string(status).decode()
        super().__init__(f"fd status {status} ({msg})" + (f": {detail}" if detail else ""))


def fd_workspace_bytes(N: int, D: int, b_max: int, m_max: int) -> int:
    return int(lib.fd_workspace_bytes(N, D, b_max, m_max))


def fd_launch_count() -> int:
    return int(lib.fd_launch_count())


def fd_version() -> int:
    return int(lib.fd_version())


def _ptr(t):
    return None if t is None else t.data_ptr()


class _NoSwitch:
    def __enter__(self):
        return None

    def __exit__(self, *exc):
        return False


_NO_SWITCH = _NoSwitch()


def _on(device: torch.device):
    """Makes `device` current for a call; costs nothing when it is current already (a small product takes about as long as the
    switch back and forth)."""
    return _NO_SWITCH if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _colmajor(rows: int, cols: int, device) -> torch.Tensor:
    """(rows x cols) float32 tensor whose storage is column-major (ld = rows)."""
    return torch.empty_strided((rows, cols), (1, rows), dtype=torch.float32, device=device)


def _ld(t: torch.Tensor) -> int:
    """Leading dimension of a column-major 2-D (or 1-D) float32 tensor."""
    if t.dim() == 1:
        return t.shape[0]
    s0, s1 = t.stride()
    assert s0 == 1, "blocks must be column-major (use .t() of a contiguous (cols, rows) tensor)"
    rows, cols = t.shape
    return s1 if cols > 1 else max(rows, s1)


class Context:
    """One data set on one GPU.  Methods mirror the C entry points one to one."""

    def __init__(self, X: torch.Tensor, b_max: int = 64, m_max: int = 0, center: bool = True, stream=None):
        assert X.is_cuda and X.dtype == torch.float32 and X.dim() == 2 and X.stride(1) == 1
        self.N, self.D = int(X.shape[0]), int(X.shape[1])
        self.device = X.device
        self.b_max, self.m_max = int(b_max), int(m_max)
        nbytes = fd_workspace_bytes(self.N, self.D, b_max, m_max)
        if nbytes == 0:
            raise FdError(FD_ERR_INVALID, "fd_workspace_bytes rejected the shape")
        self.workspace_bytes = nbytes
        with _on(self.device):
            self._ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            off = (-self._ws.data_ptr()) % 256
            self._stream = stream if stream is not None else torch.cuda.current_stream(self.device)
            h = c_void_p()
            st = lib.fd_create(byref(h), _ptr(X), self.N, self.D, X.stride(0), 1 if center else 0, b_max, m_max,
                               c_void_p(self._ws.data_ptr() + off), nbytes, c_void_p(self._stream.cuda_stream))
        if st != FD_OK:
            raise FdError(st)
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib.fd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, ok=(FD_OK,)):
        if st != FD_OK and st not in ok:
            shard = getattr(self, "_shard", None)
            if st == FD_ERR_COMM and shard is not None and shard.error is not None:
                err, shard.error = shard.error, None
                raise FdError(st, lib.fd_last_error(self._h).decode()) from err
            raise FdError(st, lib.fd_last_error(self._h).decode())
        return st

    def set_shard(self, shard):
        """Row-sharded operation (fd_set_shard): `shard` is a shard.Shard built for this context's (N, b_max), or
        None to return to unsharded operation.  The context keeps the shard (buffer and callbacks) alive."""
        if shard is not None:
            assert shard.N == self.N and shard.b_max >= self.b_max
        self._check(lib.fd_set_shard(self._h, ctypes.byref(shard.struct) if shard is not None else None))
        self._shard = shard

    def set_option(self, name: str, value: float):
        self._check(lib.fd_set_option(self._h, name.encode(), float(value)))

    def get_option(self, name: str) -> float:
        v = c_double()
        self._check(lib.fd_get_option(self._h, name.encode(), byref(v)))
        return v.value

    def beta0(self) -> float:
        v = c_double()
        self._check(lib.fd_beta0(self._h, byref(v)))
        return v.value

    def degree(self, beta: float, alpha: float, prec: int = FD_PREC_FP32):
        """Returns (q, d, s, S_off(beta), S_off(2 beta))."""
        q, d, s = (torch.empty(self.N, dtype=torch.float32, device=self.device) for _ in range(3))
        so, so2 = c_double(), c_double()
        with _on(self.device):
            self._check(lib.fd_degree(self._h, beta, alpha, prec, _ptr(q), _ptr(d), _ptr(s), byref(so), byref(so2)))
        return q, d, s, so.value, so2.value

    def synchronize(self):
        with _on(self.device):
            self._check(lib.fd_synchronize(self._h))

    def apply(self, V: torch.Tensor, out: torch.Tensor | None = None, prec: int = FD_PREC_FP32) -> torch.Tensor:
        if V.dim() == 1:
            V = V[:, None]
        b = V.shape[1]
        Y = out if out is not None else _colmajor(self.N, b, self.device)
        with _on(self.device):
            self._check(lib.fd_apply(self._h, _ptr(V), _ld(V), b, _ptr(Y), _ld(Y), prec))
        return Y

    def apply_general(self, beta: float, V: torch.Tensor | None, left=None, right=None, Xrow=None,
                      out: torch.Tensor | None = None, prec: int = FD_PREC_FP32) -> torch.Tensor:
        if V is not None and V.dim() == 1:
            V = V[:, None]
        b = 1 if V is None else V.shape[1]
        nrow = self.N if Xrow is None else int(Xrow.shape[0])
        Y = out if out is not None else _colmajor(nrow, b, self.device)
        with _on(self.device):
            self._check(lib.fd_apply_general(self._h, beta, _ptr(left), _ptr(right), _ptr(Xrow), nrow,
                                             0 if Xrow is None else Xrow.stride(0), _ptr(V),
                                             self.N if V is None else _ld(V), b, _ptr(Y), _ld(Y), prec))
        return Y

    def eigs(self, k: int, b: int, tol: float = 1e-6, max_applies: int = 1000, Q0: torch.Tensor | None = None,
             allow_not_converged: bool = False):
        """Returns (evals[k+1] float64 numpy, evecs N x (k+1) column-major tensor, info)."""
        import numpy as np
        ev = (c_double * (k + 1))()
        U = _colmajor(self.N, k + 1, self.device)
        info = fd_eigs_info()
        with _on(self.device):
            st = lib.fd_eigs(self._h, k, b, tol, max_applies, _ptr(Q0), 0 if Q0 is None else _ld(Q0),
                             0 if Q0 is None else Q0.shape[1], ev, _ptr(U), _ld(U), byref(info))
        self._check(st, ok=(FD_OK, FD_ERR_NOT_CONVERGED) if allow_not_converged else (FD_OK,))
        return np.array(ev[:], dtype=np.float64), U, info

    def beta_flow(self, k: int, b: int, alpha: float, beta_start: float = 0.0, beta_max: float = 1000.0,
                  tol: float = 1e-6, max_applies: int = 2000, warm_start: bool = True, eta: float = 0.0,
                  Q0: torch.Tensor | None = None, max_probes: int = 64):
        """Returns (beta_x, outcome name, evals, evecs, list of probe dicts)."""
        import numpy as np
        opts = fd_flow_opts(beta_start, beta_max, 2.0, alpha, eta, tol, k, b, max_applies, 1 if warm_start else 0)
        log = (fd_probe * max_probes)()
        n = c_int32(max_probes)
        outcome = c_int32()
        bx = c_double()
        ev = (c_double * (k + 1))()
        U = _colmajor(self.N, k + 1, self.device)
        with _on(self.device):
            st = lib.fd_beta_flow(self._h, byref(opts), _ptr(Q0), 0 if Q0 is None else _ld(Q0),
                                  0 if Q0 is None else Q0.shape[1], log, byref(n), byref(outcome), byref(bx), ev,
                                  _ptr(U), _ld(U))
        self._check(st)
        recs = [{f[0]: getattr(log[i], f[0]) for f in fd_probe._fields_} for i in range(n.value)]
        return bx.value, FLOW_OUTCOMES[outcome.value], np.array(ev[:], dtype=np.float64), U, recs

    def beta_flow_cascade(self, k: int, b: int, alpha: float, stages, beta_start: float = 0.0, beta_max: float = 1000.0,
                          max_applies: int = 2000, warm_start: bool = True, Q0: torch.Tensor | None = None,
                          max_probes: int = 64):
        """stages: sequence of (precision, eta, tol) with eta / tol <= 0 for the mode's defaults.
        Returns (beta_x, outcome name, evals, evecs, [list of probe dicts per stage])."""
        import numpy as np
        opts = fd_flow_opts(beta_start, beta_max, 2.0, alpha, 0.0, 0.0, k, b, max_applies, 1 if warm_start else 0)
        ns = len(stages)
        st_arr = (fd_cascade_stage * ns)(*[fd_cascade_stage(int(p), float(e), float(t)) for p, e, t in stages])
        cap = max_probes * ns
        log = (fd_probe * cap)()
        n = c_int32(cap)
        first = (c_int32 * (ns + 1))()
        outcome = c_int32()
        bx = c_double()
        ev = (c_double * (k + 1))()
        U = _colmajor(self.N, k + 1, self.device)
        with _on(self.device):
            st = lib.fd_beta_flow_cascade(self._h, byref(opts), st_arr, ns, _ptr(Q0), 0 if Q0 is None else _ld(Q0),
                                          0 if Q0 is None else Q0.shape[1], log, byref(n), first, byref(outcome), byref(bx),
                                          ev, _ptr(U), _ld(U))
        self._check(st)
        recs = [[{f[0]: getattr(log[i], f[0]) for f in fd_probe._fields_} for i in range(first[s], first[s + 1])]
                for s in range(ns)]
        return bx.value, FLOW_OUTCOMES[outcome.value], np.array(ev[:], dtype=np.float64), U, recs

    def nystrom(self, Xnew: torch.Tensor, psi: torch.Tensor, evals) -> torch.Tensor:
        m = psi.shape[1]
        lam = (c_double * m)(*[float(v) for v in evals])
        out = _colmajor(int(Xnew.shape[0]), m, self.device)
        with _on(self.device):
            self._check(lib.fd_nystrom(self._h, _ptr(Xnew), Xnew.shape[0], Xnew.stride(0), _ptr(psi), _ld(psi), m, lam,
                                       _ptr(out), _ld(out)))
        return out

    def ladder_start(self, old: "Context", Xnew: torch.Tensor, evecs_old: torch.Tensor, evals) -> torch.Tensor:
        """Warm-start basis for this (new, larger) level from the eigenpairs of `old` (the level over its first rows)."""
        m = evecs_old.shape[1]
        lam = (c_double * m)(*[float(v) for v in evals])
        Q0 = _colmajor(self.N, m, self.device)
        with _on(self.device):
            self._check(lib.fd_ladder_start(old._h, self._h, _ptr(Xnew), Xnew.stride(0), _ptr(evecs_old), _ld(evecs_old), m,
                                            lam, _ptr(Q0), _ld(Q0)))
        return Q0

    def scale_by_degree(self, v: torch.Tensor, power: float) -> torch.Tensor:
        out = _colmajor(self.N, v.shape[1], self.device)
        with _on(self.device):
            self._check(lib.fd_scale_by_degree(self._h, _ptr(v), _ld(v), v.shape[1], power, _ptr(out), _ld(out)))
        return out


FD_STATIC_MAX_N, FD_STATIC_MAX_D, FD_STATIC_MAX_B = 8192, 32, 32


def fd_apply_general_static(X: torch.Tensor, beta: float, V: torch.Tensor, left=None, right=None,
                            out: torch.Tensor | None = None) -> torch.Tensor:
    """Y = diag(left) K(X, X) diag(right) V through the entry point that allocates nothing on the device: its
    scratch is the library's own fixed device array.  For callers that cannot allocate; sizes are limited to
    FD_STATIC_MAX_N / _D / _B, and calls must not overlap on the GPU.  `out` must be given by such a caller; when it
    is omitted here the binding allocates it for convenience (that allocation is the binding's, not the library's)."""
    assert X.is_cuda and X.dtype == torch.float32 and X.dim() == 2 and X.stride(1) == 1
    if V.dim() == 1:
        V = V[:, None]
    N, D, b = int(X.shape[0]), int(X.shape[1]), int(V.shape[1])
    Y = out if out is not None else _colmajor(N, b, X.device)
    err = ctypes.create_string_buffer(256)
    with _on(X.device):
        st = lib.fd_apply_general_static(_ptr(X), N, D, X.stride(0), float(beta), _ptr(left), _ptr(right), _ptr(V), _ld(V), b,
                                         _ptr(Y), _ld(Y), c_void_p(torch.cuda.current_stream(X.device).cuda_stream), err, 256)
    if st != FD_OK:
        raise FdError(st, err.value.decode())
    return Y


# ---- kept keys and values, rotary positions (fd.h: "kept keys and values") ------------------------------------------
_DTYPES = {torch.bfloat16: FD_BF16, torch.float16: FD_FP16, torch.float32: FD_FP32}
_LAYOUTS = {"half": FD_ROTARY_HALF, "interleaved": FD_ROTARY_INTERLEAVED}
_SCALINGS = {"none": FD_ROTARY_PLAIN, "linear": FD_ROTARY_LINEAR, "base": FD_ROTARY_BASE, "ramp": FD_ROTARY_RAMP}


def _refuse(what: str):
    raise FdError(FD_ERR_INVALID, what)


def _need(cond, what: str):
    if not cond:
        _refuse(what)


# These checks and the calls below run once per operator and decoding step, some in less time than the kernel they launch.  So texts are made where a check
# fails, and the structures of fd.h are packed in one step (fd_heads, fd_kv_append_args, fd_kv_attend_args, fd_kv_evict_args; the test-suite holds the
# formats against the ctypes structures of the same names).
_HEADS = struct.Struct("@Pqqi4x")
_APPEND = struct.Struct("@" + "Pqqi4x" * 4 + "PPdii")
_ATTEND = struct.Struct("@" + "Pqqi4x" * 2 + "diiPPPq")
_EVICT = struct.Struct("@PPqPqiiiiPP")
_NO_HEADS = (0, 0, 0, 0)


def _need_tensor(t, dtype, dims: int, index: int, what: str):
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != dims or t.get_device() != index:
        _refuse(f"{what}: a {dims}-d {dtype} tensor on cuda:{index}")


def _heads(t: torch.Tensor, dtype, index: int, head_dim: int, tokens: int, what: str):
    """[tokens, heads, head_dim] with unit stride inside a head, as the fields of an fd_heads; strides of single tokens and heads do not matter."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != 3 or t.get_device() != index:
        _refuse(f"{what}: a 3-d {dtype} tensor on cuda:{index}")
    n, h, d = t.shape
    st, sh, sd = t.stride()
    if n != tokens or d != head_dim or (sd != 1 and d != 1):
        _refuse(f"{what}: [{tokens}, heads, {head_dim}] with unit stride inside a head")
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(f"{what} requires a gradient, and no graph is built here: call under torch.no_grad() (the gradient of fd_rotary is fd_rotary with inverse=True)")
    return t.data_ptr(), st if n > 1 else h * d, sh if h > 1 else d, h


def _table(t: torch.Tensor, what: str):
    """(stride, pages) of the rows of a page table; rows may lie in any distance, 0 (one row for all sequences, an expanded tensor) included."""
    rows, cols = t.shape
    row, unit = t.stride()
    if unit != 1 and cols != 1:
        _refuse(f"{what}: [batch, pages], unit stride inside a row")
    return row if rows > 1 else cols, cols


class _Messages(threading.local):
    def __init__(self):
        self.buf = ctypes.create_string_buffer(256)


_messages = _Messages()


def _call(index: int, fn, *args):
    """fn(*args, current stream, errbuf, its length) on a device."""
    err = _messages.buf
    if torch._C._cuda_getDevice() == index:
        st = fn(*args, torch._C._cuda_getCurrentRawStream(index), err, 256)
    else:
        with torch.cuda.device(index):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(index), err, 256)
    if st != FD_OK:
        raise FdError(st, err.value.decode())


def fd_rotary_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                          original_len: float = 0.0, lo: float = 1.0, hi: float = 32.0, device=None) -> torch.Tensor:
    """Frequencies of rotary positions (rot_dim / 2 doubles) on `device`; scaling: "none", "linear", "base" or "ramp"."""
    _need(scaling in _SCALINGS, f"scaling: one of {sorted(_SCALINGS)}")
    out = (c_double * max(1, rot_dim // 2))()
    st = lib.fd_rotary_frequencies(rot_dim, base, _SCALINGS[scaling], factor, original_len, lo, hi, out)
    if st != FD_OK:
        raise FdError(st, "rot_dim, base, factor or ramp out of range")
    return torch.tensor(list(out), dtype=torch.float64, device=device)


def _rotary_args(positions, freqs, tokens: int, index: int, layout: str):
    _need_tensor(positions, torch.int32, 1, index, "positions")
    _need_tensor(freqs, torch.float64, 1, index, "freqs")
    if positions.numel() != tokens or not positions.is_contiguous():
        _refuse(f"positions: {tokens} contiguous values")
    if not freqs.is_contiguous():
        _refuse("freqs must be contiguous")
    code = _LAYOUTS.get(layout)
    return code if code is not None else _refuse(f"layout: one of {sorted(_LAYOUTS)}")


def fd_rotary(x: torch.Tensor, positions: torch.Tensor, freqs: torch.Tensor, layout: str = "half", scale: float = 1.0,
              inverse: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """Rotary positions of x [tokens, heads, head_dim] on the current stream; with `inverse` the transpose, which takes the gradient of the
    result to the gradient of x.  `out` may be x.  No graph is built: a tensor that requires a gradient is refused outside torch.no_grad()."""
    dt = x.dtype if isinstance(x, torch.Tensor) else None
    code = _DTYPES.get(dt)
    if code is None or not x.is_cuda or x.dim() != 3:
        _refuse("x: a CUDA tensor [tokens, heads, head_dim] of bf16, fp16 or fp32")
    index = x.get_device()
    tokens, _, d = x.shape
    order = _rotary_args(positions, freqs, tokens, index, layout)
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else out
    _call(index, lib.fd_rotary, _HEADS.pack(*_heads(x, dt, index, d, tokens, "x")), _HEADS.pack(*_heads(y, dt, index, d, tokens, "out")), code, tokens, d,
          positions.data_ptr(), freqs.data_ptr(), 2 * freqs.numel(), order, scale, 1 if inverse else 0)
    return y


class KVBatch:
    """The sequences of a call: page table [batch, pages], tokens in the cache (the new ones among them) [batch], first new token of each
    [batch + 1], all int32 on the GPU and read there (a captured call takes their values at replay), and upper bounds of the new tokens in
    all, of one sequence's new tokens and of a sequence's length."""

    def __init__(self, page_table: torch.Tensor, kv_len: torch.Tensor, q_start: torch.Tensor, total_q: int, max_new: int, max_len: int):
        dev = page_table.device
        _need(page_table.is_cuda, "page_table: a CUDA tensor")
        _need_tensor(page_table, torch.int32, 2, dev.index, "page_table")
        _need_tensor(kv_len, torch.int32, 1, dev.index, "kv_len")
        _need_tensor(q_start, torch.int32, 1, dev.index, "q_start")
        n = page_table.shape[0]
        stride, cols = _table(page_table, "page_table")
        _need(all(0 <= x < 1 << 31 for x in (total_q, max_new, max_len)), "total_q, max_new, max_len: 0 to 2^31 - 1")       # (fields of 32 bits would wrap)
        _need(kv_len.shape[0] == n and q_start.shape[0] == n + 1 and kv_len.is_contiguous() and q_start.is_contiguous(),
              f"kv_len: {n} contiguous values, q_start: {n + 1}")
        self.device, self.total_q = dev, int(total_q)
        self.page_table, self.kv_len, self.q_start = page_table, kv_len, q_start
        self.batch, self.max_len = n, int(max_len)
        self.struct = fd_kv_batch(page_table.data_ptr(), stride, kv_len.data_ptr(), q_start.data_ptr(), n, cols, total_q, max_new, max_len)
        self.ref = byref(self.struct)


class KVCache:
    """Keys and values in pages: two pools [page, token in page, head, head_dim] (any strides with unit stride inside a head, so a pool laid
    out [page, head, token, head_dim] is passed transposed).  Calls run on the current stream and mirror the C entry points; workspaces are
    taken from the current stream's allocator for each call, so calls on several streams and captured graphs share nothing but the pools.  No graph is
    built: tensors that require a gradient are refused outside torch.no_grad().  A cache has to outlive its calls and the graphs that hold them."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        _need(isinstance(k_pages, torch.Tensor) and k_pages.is_cuda and k_pages.dim() == 4 and k_pages.dtype in (torch.bfloat16, torch.float16),
              "k_pages: a CUDA tensor [page, token, head, head_dim] of bf16 or fp16")
        dev = k_pages.device
        _need_tensor(v_pages, k_pages.dtype, 4, dev.index, "v_pages")
        _need(k_pages.shape == v_pages.shape and k_pages.stride(3) == 1 and v_pages.stride(3) == 1, "k_pages, v_pages: equal shapes, unit stride inside a head")
        _need(not ((k_pages.requires_grad or v_pages.requires_grad) and torch.is_grad_enabled()), "k_pages, v_pages require a gradient, and no graph is built here")
        self.device, self.dtype = dev, k_pages.dtype
        self.k_pages, self.v_pages = k_pages, v_pages
        pages, size, heads, d = k_pages.shape
        self.heads, self.head_dim = heads, d
        self._status = torch.zeros(4, dtype=torch.int32, device=dev)
        desc = fd_kv_desc(k_pages.data_ptr(), v_pages.data_ptr(), *[t.stride(i) if t.shape[i] > 1 else t.shape[1] * t.shape[2] * d
                                                                   for t in (k_pages, v_pages) for i in (0, 1, 2)],
                          pages, size, heads, d, _DTYPES[k_pages.dtype], self._status.data_ptr())
        h, err = c_void_p(), ctypes.create_string_buffer(256)
        with _on(dev):
            torch.cuda.current_stream(dev).synchronize()       # the status words are zero for every stream from here on
            st = lib.fd_kv_create(byref(h), byref(desc), err, 256)
        if st != FD_OK:
            raise FdError(st, err.value.decode())
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib.fd_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def synchronize(self):
        """Waits for the current stream; raises FdError if a page number or length was out of range, or a bounded wait ran out."""
        with _on(self.device):
            st = lib.fd_kv_synchronize(self._h, torch._C._cuda_getCurrentRawStream(self.device.index))
        if st != FD_OK:
            raise FdError(st, "a page number or a length was out of range" if st == FD_ERR_INVALID else "")

    def _batch(self, batch: KVBatch):
        if batch.device != self.device:
            _refuse(f"the batch is on {batch.device}, the cache on {self.device}")
        return batch.ref

    def append(self, batch: KVBatch, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor | None = None, freqs: torch.Tensor | None = None,
               layout: str = "half", scale: float = 1.0, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None):
        """Writes the new tokens' keys (rotated, if there are positions) and values into the cache; rotates q beside them and returns it."""
        n, index, dt, d = batch.total_q, self.device.index, self.dtype, self.head_dim
        ref = self._batch(batch)
        rot, hq, ho = (0, 0, scale, 0, 0), _NO_HEADS, _NO_HEADS
        if positions is not None:
            order = _rotary_args(positions, freqs, n, index, layout)
            rot = (positions.data_ptr(), freqs.data_ptr(), scale, 2 * freqs.numel(), order)
        if q is not None:
            hq = _heads(q, dt, index, d, n, "q")
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            ho = _heads(q_out, dt, index, d, n, "q_out")
        _call(index, lib.fd_kv_append, self._h, ref, _APPEND.pack(*_heads(k, dt, index, d, n, "k"), *_heads(v, dt, index, d, n, "v"), *hq, *ho, *rot))
        return q_out

    def attend(self, batch: KVBatch, q: torch.Tensor, scale: float | None = None, causal: bool = True, window: int = 0,
               out: torch.Tensor | None = None, lse: torch.Tensor | None = None, weights: torch.Tensor | None = None,
               weights_out: torch.Tensor | None = None):
        """Returns (out, lse) for the new tokens' queries [total_q, query heads, head_dim]; scale defaults to head_dim^-1/2.  With `weights`
        ([batch, heads, >= max_len] fp32) and / or `weights_out` (default: weights itself) the softmax weights that every cached token received are
        added up: weights_out = weights (or 0) + their sum."""
        n, index, dt, d = batch.total_q, self.device.index, self.dtype, self.head_dim
        ref = self._batch(batch)
        hq = _heads(q, dt, index, d, n, "q")
        heads = hq[3]
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        if lse is None:
            lse = torch.empty((n, heads), dtype=torch.float32, device=self.device)
        else:
            _need_tensor(lse, torch.float32, 2, index, "lse")
            if lse.shape != (n, heads) or not lse.is_contiguous():
                _refuse("lse: [total_q, query heads], contiguous")
        w_in = w_out = w_stride = 0
        if weights is not None or weights_out is not None:
            if weights_out is None:
                weights_out = weights
            w_stride = self._check_weights(weights_out, batch)
            w_out = weights_out.data_ptr()
            if weights is not None:
                if self._check_weights(weights, batch) != w_stride:
                    _refuse("weights and weights_out: equal shapes")
                w_in = weights.data_ptr()
        size = lib.fd_kv_attend_bytes(self._h, ref, heads, 1 if w_out else 0)
        ws = torch.empty(size, dtype=torch.uint8, device=self.device) if size else None
        _call(index, lib.fd_kv_attend, self._h, ref, _ATTEND.pack(*hq, *_heads(out, dt, index, d, n, "out"), d ** -0.5 if scale is None else scale,
                                                                 1 if causal else 0, window or 0, lse.data_ptr(), w_in, w_out, w_stride),
              None if ws is None else ws.data_ptr(), size)
        return out, lse

    def _check_weights(self, t: torch.Tensor, batch: KVBatch) -> int:
        _need_tensor(t, torch.float32, 3, self.device.index, "weights")
        if t.requires_grad and torch.is_grad_enabled():
            _refuse("weights require a gradient, and no graph is built here")
        n, h, length = t.shape
        if n != batch.batch or h != self.heads or length < batch.max_len or not t.is_contiguous():
            _refuse(f"weights: [{batch.batch}, {self.heads}, {batch.max_len} or more], contiguous")
        return length

    def evict(self, batch: KVBatch, weights: torch.Tensor, keep: int, first: int = 0, recent: int = 0, new_table: torch.Tensor | None = None,
              kept: torch.Tensor | None = None, new_len: torch.Tensor | None = None, weights_out: torch.Tensor | None = None):
        """Every head keeps `keep` tokens of each longer sequence: the first, the recent and the heaviest of the others, in order, moved to
        the front of the sequence's pages (or to new_table's).  Returns (kept slots [batch, heads, keep], new lengths, weights)."""
        index, ref = self.device.index, self._batch(batch)
        w_stride = self._check_weights(weights, batch)
        if weights_out is None:
            weights_out = weights
        elif self._check_weights(weights_out, batch) != w_stride:
            _refuse("weights and weights_out: equal shapes")
        table = batch.page_table if new_table is None else new_table
        _need_tensor(table, torch.int32, 2, index, "new_table")
        stride, cols = _table(table, "new_table")
        if table.shape[0] != batch.batch:
            _refuse(f"new_table: {batch.batch} rows")
        if kept is None:
            kept = torch.empty((batch.batch, self.heads, max(keep, 0)), dtype=torch.int32, device=self.device)
        if new_len is None:
            new_len = torch.empty(batch.batch, dtype=torch.int32, device=self.device)
        _need_tensor(kept, torch.int32, 3, index, "kept")
        _need_tensor(new_len, torch.int32, 1, index, "new_len")
        if kept.shape != (batch.batch, self.heads, keep) or not kept.is_contiguous():
            _refuse(f"kept: [{batch.batch}, {self.heads}, {keep}], contiguous")
        if new_len.numel() != batch.batch or not new_len.is_contiguous():
            _refuse(f"new_len: {batch.batch} contiguous values")
        _call(index, lib.fd_kv_evict, self._h, ref, _EVICT.pack(weights.data_ptr(), weights_out.data_ptr(), w_stride, table.data_ptr(), stride, cols,
                                                                keep, first, recent, kept.data_ptr(), new_len.data_ptr()))
        return kept, new_len, weights_out


def fd_unit_peaks(device) -> dict:
    """Measured unit throughput of `device` (fd.h: fd_unit_peaks): rates per clock per SM and SM cycles per tcgen05.mma."""
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device=device)
    out = fd_unit_rates()
    with torch.cuda.device(device):
        st = lib.fd_unit_peaks(_ptr(scratch), scratch.numel(), c_void_p(torch.cuda.current_stream(device).cuda_stream),
                               ctypes.byref(out))
    if st != FD_OK:
        raise FdError(st)
    return {n: getattr(out, n) for n, _ in fd_unit_rates._fields_}


def to_colmajor(a, device) -> torch.Tensor:
    """numpy (rows x cols) array -> column-major float32 device tensor."""
    import numpy as np
    a = np.asarray(a, dtype=np.float32)
    if a.ndim == 1:
        a = a[:, None]
    t = torch.from_numpy(np.ascontiguousarray(a.T)).to(device)
    return t.t()
