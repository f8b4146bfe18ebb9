"""ctypes binding of libcovspec.so (declared in include/covspec.h).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.  PyTorch is
used for device memory and the current stream.  There is no CPU fallback: loading fails loudly
when the compiled library is missing, and every call raises on a non-zero status.
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import os
import warnings
from typing import Optional

import numpy as np
import torch

# COVSPEC_LIBRARY selects another build of the same library (the checked one, libcovspec_debug.so)
_LIB_PATH = os.environ.get("COVSPEC_LIBRARY") or \
    os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcovspec.so")

COVSPEC_F32, COVSPEC_BF16, COVSPEC_F16, COVSPEC_E4M3, COVSPEC_INT8 = 0, 1, 2, 3, 4
NORM_MODES = {"minmax": 0, "zscore": 1, "none": 2}
HEAD_REDUCE = {"max": 0, "mean": 1}

EXPORTS = [
    "covspec_default_config", "covspec_budgets", "covspec_plan_sizes", "covspec_prune_init",
    "covspec_prune_destroy", "covspec_workspace_bytes", "covspec_score", "covspec_select",
    "covspec_compact", "covspec_compact_rows", "covspec_prune", "covspec_get_device_status",
    "covspec_last_launch_count", "covspec_strerror", "covspec_last_cuda_error",
    "covspec_profile_begin", "covspec_profile_end", "covspec_profile_stage_count",
    "covspec_profile_stage_name", "covspec_query_score_static", "covspec_selftest_wait_timeout",
    "covspec_correct", "covspec_fanout", "covspec_branch_candidates", "covspec_branch_candidates_host",
    "covspec_uplink_bits", "covspec_downlink_bits", "covspec_comm_latency", "covspec_ema_update",
    "covspec_draft_length", "covspec_get_iteration_counts", "covspec_build_has_bounds_checks",
    "covspec_selftest_fill_workspace", "covspec_selftest_static_timeout",
    "covspec_cache_write", "covspec_cache_read", "covspec_cache_attend", "covspec_cache_attend_workspace",
    "covspec_edit_logits", "covspec_selftest_attend_timeout",
]
STATIC_MAX_BATCH = 256
STATIC_MAX_QUERY_ELEMS = 1 << 20


class Config(C.Structure):
    _fields_ = [
        ("dtype", C.c_int), ("d", C.c_int), ("n_heads", C.c_int), ("head_dim", C.c_int),
        ("act_layers", C.c_int), ("lam", C.c_float), ("norm_mode", C.c_int),
        ("head_reduce", C.c_int), ("presel_factor", C.c_float), ("rank_frac", C.c_float),
        ("rank_cap", C.c_int), ("eig_iters", C.c_int), ("eig_oversample", C.c_int),
        ("max_batch", C.c_int), ("max_total_vis", C.c_longlong), ("max_total_txt", C.c_longlong),
        ("max_vis_per_req", C.c_int), ("max_presel_per_req", C.c_int),
        ("max_total_presel", C.c_longlong), ("relevance_path", C.c_int), ("lowrank_mode", C.c_int),
        ("ritz_window", C.c_int), ("activity_overlap", C.c_int), ("conv_tol", C.c_float),
        ("eig_early_stop", C.c_int),
    ]


class Problem(C.Structure):
    _fields_ = [
        ("batch", C.c_int), ("X", C.c_void_p), ("vis_offsets", C.POINTER(C.c_int)),
        ("Q", C.c_void_p), ("txt_offsets", C.POINTER(C.c_int)), ("Wq", C.c_void_p),
        ("Wk", C.c_void_p), ("Hs", C.POINTER(C.c_void_p)), ("keep", C.POINTER(C.c_int)),
        ("keep_ratio", C.c_double),
    ]


class Cache(C.Structure):
    _fields_ = [
        ("store", C.c_int), ("pages", C.c_int), ("heads", C.c_int), ("page_size", C.c_int), ("head_dim", C.c_int),
        ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
        ("k_page_stride", C.c_longlong), ("v_page_stride", C.c_longlong),
    ]


class Tokens(C.Structure):
    _fields_ = [
        ("batch", C.c_int), ("offsets", C.c_void_p), ("lengths", C.c_void_p), ("table", C.c_void_p),
        ("table_width", C.c_int), ("table_stride", C.c_longlong),
    ]


class Edits(C.Structure):
    _fields_ = [
        ("batch", C.c_int), ("row_offsets", C.c_void_p), ("history", C.c_void_p), ("history_offsets", C.c_void_p),
        ("history_len", C.c_int), ("prompt_lengths", C.c_void_p), ("drafted", C.c_void_p), ("repetition", C.c_void_p),
        ("presence", C.c_void_p), ("frequency", C.c_void_p), ("bias_ids", C.c_void_p), ("bias_values", C.c_void_p),
        ("bias_offsets", C.c_void_p), ("bias_len", C.c_int), ("mask", C.c_void_p), ("mask_stride", C.c_longlong),
    ]


class CovspecError(RuntimeError):
    def __init__(self, status, where):
        lib = load_library()
        msg = lib.covspec_strerror(status).decode()
        if status == -5:
            msg += " (" + lib.covspec_last_cuda_error().decode() + ")"
        super().__init__(f"{where}: {msg} [{status}]")
        self.status = status


_lib = None


def load_library():
    """Loads libcovspec.so (built by paper_2605_02218_b200.build).  Raises if it is missing."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} not found: build it with `python -m paper_2605_02218_b200.build` "
            "(there is no fallback path)")
    lib = C.CDLL(_LIB_PATH)
    vp, ip, fp = C.c_void_p, C.POINTER(C.c_int), C.c_void_p
    lib.covspec_default_config.argtypes = [C.POINTER(Config)]
    lib.covspec_default_config.restype = None
    lib.covspec_budgets.argtypes = [C.POINTER(Config), C.c_int, C.c_int, ip, ip, ip]
    lib.covspec_plan_sizes.argtypes = [C.POINTER(Config), C.POINTER(Problem), ip, ip]
    lib.covspec_prune_init.argtypes = [C.POINTER(Config), C.POINTER(vp)]
    lib.covspec_prune_destroy.argtypes = [vp]
    lib.covspec_workspace_bytes.argtypes = [vp]
    lib.covspec_workspace_bytes.restype = C.c_longlong
    lib.covspec_score.argtypes = [vp, C.POINTER(Problem), fp, fp, fp, vp]
    lib.covspec_select.argtypes = [vp, C.POINTER(Problem), fp, vp, ip, vp, fp, vp]
    lib.covspec_compact.argtypes = [vp, C.POINTER(Problem), vp, ip, vp, vp, vp]
    lib.covspec_prune.argtypes = [vp, C.POINTER(Problem), vp, vp, ip, vp]
    lib.covspec_compact_rows.argtypes = [vp, C.POINTER(Problem), vp, ip, vp, C.c_longlong, vp, vp]
    lib.covspec_get_device_status.argtypes = [vp, vp]
    lib.covspec_selftest_wait_timeout.argtypes = [vp, vp]
    lib.covspec_selftest_fill_workspace.argtypes = [vp, C.c_int, vp]
    lib.covspec_get_iteration_counts.argtypes = [vp, C.c_int, ip, vp]
    lib.covspec_fanout.argtypes = [C.c_int, C.c_double, C.c_int]
    lib.covspec_uplink_bits.argtypes = [C.c_longlong, C.c_int, C.c_longlong, C.c_int]
    lib.covspec_uplink_bits.restype = C.c_double
    lib.covspec_downlink_bits.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.c_longlong, C.c_int]
    lib.covspec_downlink_bits.restype = C.c_double
    lib.covspec_comm_latency.argtypes = [C.c_double, C.c_double, C.c_double]
    lib.covspec_comm_latency.restype = C.c_double
    lib.covspec_ema_update.argtypes = [C.c_double, C.c_double, C.c_int, C.c_int]
    lib.covspec_ema_update.restype = C.c_double
    lib.covspec_draft_length.argtypes = [C.c_int] + [C.c_double] * 6 + [C.c_int, C.c_int]
    lib.covspec_branch_candidates.argtypes = [C.c_int, C.c_int, C.c_int, C.c_longlong, vp, vp, vp, C.c_int, vp, vp]
    lib.covspec_branch_candidates_host.argtypes = lib.covspec_branch_candidates.argtypes
    lib.covspec_correct.argtypes = [C.c_int, C.c_int, C.c_int, C.c_longlong, vp, vp, vp, vp, C.c_float,
                                    vp, vp, vp, vp, vp, vp]
    lib.covspec_last_launch_count.argtypes = [vp]
    lib.covspec_strerror.argtypes = [C.c_int]
    lib.covspec_strerror.restype = C.c_char_p
    lib.covspec_last_cuda_error.argtypes = []
    lib.covspec_last_cuda_error.restype = C.c_char_p
    lib.covspec_query_score_static.argtypes = [C.c_int, C.c_int, C.c_int, vp, ip, vp, ip, fp, vp]
    lib.covspec_selftest_static_timeout.argtypes = [C.c_int, C.c_int, vp, ip, vp, ip, fp, vp]
    lib.covspec_profile_begin.argtypes = [vp, C.c_int]
    lib.covspec_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.c_int, ip]
    lib.covspec_profile_stage_count.argtypes = []
    lib.covspec_profile_stage_name.argtypes = [C.c_int]
    lib.covspec_profile_stage_name.restype = C.c_char_p
    cp, tp, ll = C.POINTER(Cache), C.POINTER(Tokens), C.c_longlong
    lib.covspec_cache_write.argtypes = [cp, tp, C.c_int, C.c_int, vp, vp, ll, ll, vp, vp, C.c_int, vp]
    lib.covspec_cache_read.argtypes = [cp, tp, C.c_int, C.c_int, vp, vp, vp]
    lib.covspec_cache_attend.argtypes = [cp, tp, C.c_int, C.c_int, vp, ll, C.c_int, C.c_float, C.c_int, C.c_int, vp, ll, vp, vp,
                                         ll, vp]
    lib.covspec_selftest_attend_timeout.argtypes = lib.covspec_cache_attend.argtypes[:-1] + [C.c_int, C.c_int, vp]
    lib.covspec_cache_attend_workspace.argtypes = [cp, C.c_int]
    lib.covspec_cache_attend_workspace.restype = ll
    lib.covspec_edit_logits.argtypes = [C.c_int, C.c_int, C.c_int, ll, vp, vp, C.POINTER(Edits), vp]
    from .build import binding_path
    _native = _load_native(lib, binding_path())
    _lib = lib
    return lib


_native = None


def _load_native(lib, path: str):
    """The native part of the binding with the library's functions given to it, or None: the calls that it makes shorter then
    go through ctypes."""
    if not os.path.exists(path):
        return None
    try:
        loader = importlib.machinery.ExtensionFileLoader(__package__ + "._binding", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader(loader.name, loader))
        loader.exec_module(module)
    except ImportError as e:
        warnings.warn(f"{path} does not load, calls go through ctypes (build it again with "
                      f"`python -m paper_2605_02218_b200.build`): {e}", RuntimeWarning)
        return None
    module.bind(*(C.cast(f, C.c_void_p).value for f in
                  (lib.covspec_correct, lib.covspec_branch_candidates_host, lib.covspec_query_score_static, lib.covspec_cache_write,
                   lib.covspec_cache_read, lib.covspec_cache_attend, lib.covspec_edit_logits)))
    return module


def default_config(**overrides) -> Config:
    cfg = Config()
    load_library().covspec_default_config(C.byref(cfg))
    for k, v in overrides.items():
        if k == "lambda_":
            k = "lam"
        if k == "norm_mode" and isinstance(v, str):
            v = NORM_MODES[v]
        if k == "head_reduce" and isinstance(v, str):
            v = HEAD_REDUCE[v]
        if not hasattr(cfg, k):
            raise KeyError(k)
        setattr(cfg, k, v)
    return cfg


def budgets(cfg: Config, n: int, keep: int):
    b, m, r = C.c_int(), C.c_int(), C.c_int()
    st = load_library().covspec_budgets(C.byref(cfg), n, keep, C.byref(b), C.byref(m), C.byref(r))
    if st:
        raise CovspecError(st, "covspec_budgets")
    return b.value, m.value, r.value


def _i32(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(C.c_int))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


class _Marshalled:
    """Keeps the host arrays referenced by a Problem alive."""

    def __init__(self, X, Q, vis_offsets, txt_offsets, Wq=None, Wk=None, Hs=None, keep=None,
                 keep_ratio=0.0):
        self.tensors = (X, Q, Wq, Wk, Hs)
        for t in (X, Q, Wq, Wk) + tuple(Hs or ()):
            if t is not None:
                assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors required"
        self.vis, vis_p = _i32(vis_offsets)
        self.txt, txt_p = _i32(txt_offsets)
        self.batch = len(self.vis) - 1
        keep_p = None
        if keep is not None:
            self.keep, keep_p = _i32(keep)
        hs_p = None
        if Hs:
            self.hs = (C.c_void_p * len(Hs))(*[h.data_ptr() for h in Hs])
            hs_p = C.cast(self.hs, C.POINTER(C.c_void_p))
        self.problem = Problem(self.batch, _ptr(X), vis_p, _ptr(Q), txt_p, _ptr(Wq), _ptr(Wk), hs_p,
                               keep_p, float(keep_ratio))


# torch's own accessors of the current stream's address; a build without them takes the public route
_raw_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_of_device = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _raw_stream() -> int:
    """The address torch.cuda.current_stream().cuda_stream gives, without making the Stream object (0.2 us
    against 3.2)."""
    if _raw_device is None or _raw_of_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_of_device(_raw_device())


def _stream():
    return C.c_void_p(_raw_stream())


class Pruner:
    """One context (workspace + plan cache) for a fixed configuration and capacity."""

    def __init__(self, cfg: Config):
        self.lib = load_library()
        self.cfg = cfg
        self._ctx = C.c_void_p()
        st = self.lib.covspec_prune_init(C.byref(cfg), C.byref(self._ctx))
        if st:
            raise CovspecError(st, "covspec_prune_init")
        self._keepalive = None

    @classmethod
    def for_workload(cls, wl, **overrides) -> "Pruner":
        """Context sized exactly for a workloads.Workload."""
        lib = load_library()
        cfg = default_config(
            dtype=COVSPEC_BF16 if wl.dtype == torch.bfloat16 else COVSPEC_F32, d=wl.d,
            n_heads=wl.n_heads, head_dim=wl.head_dim if wl.n_heads else 0,
            act_layers=wl.act_layers, lam=wl.lam, **overrides)
        n = np.diff(wl.vis_offsets)
        cfg.max_batch = wl.batch
        cfg.max_total_vis = int(wl.vis_offsets[-1])
        cfg.max_total_txt = int(wl.txt_offsets[-1])
        cfg.max_vis_per_req = int(n.max())
        vis, vis_p = _i32(wl.vis_offsets)
        txt, txt_p = _i32(wl.txt_offsets)
        keep, keep_p = _i32(wl.keep)
        prob = Problem(wl.batch, None, vis_p, None, txt_p, None, None, None, keep_p, 0.0)
        po = np.zeros(wl.batch + 1, dtype=np.int32)
        st = lib.covspec_plan_sizes(C.byref(cfg), C.byref(prob), None,
                                    po.ctypes.data_as(C.POINTER(C.c_int)))
        if st:
            raise CovspecError(st, "covspec_plan_sizes")
        cfg.max_total_presel = int(po[-1])
        cfg.max_presel_per_req = int(np.diff(po).max())
        return cls(cfg)

    def close(self):
        if self._ctx:
            self.lib.covspec_prune_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def workspace_bytes(self) -> int:
        return int(self.lib.covspec_workspace_bytes(self._ctx))

    @property
    def last_launch_count(self) -> int:
        return int(self.lib.covspec_last_launch_count(self._ctx))

    def plan_sizes(self, m: _Marshalled):
        ko = np.zeros(m.batch + 1, dtype=np.int32)
        po = np.zeros(m.batch + 1, dtype=np.int32)
        st = self.lib.covspec_plan_sizes(C.byref(self.cfg), C.byref(m.problem),
                                         ko.ctypes.data_as(C.POINTER(C.c_int)),
                                         po.ctypes.data_as(C.POINTER(C.c_int)))
        if st:
            raise CovspecError(st, "covspec_plan_sizes")
        return ko, po

    def marshal(self, wl=None, **kw) -> _Marshalled:
        if wl is not None:
            kw = dict(X=wl.X, Q=wl.Q, vis_offsets=wl.vis_offsets, txt_offsets=wl.txt_offsets,
                      Wq=wl.Wq, Wk=wl.Wk, Hs=wl.Hs, keep=wl.keep)
        return _Marshalled(**kw)

    # ---- the entry points --------------------------------------------------------------------
    def score(self, m: _Marshalled):
        """covspec_score: returns (s_query, s_act, s_fused) float32 device tensors."""
        n = int(m.vis[-1])
        dev = m.tensors[0].device
        sq = torch.empty(n, dtype=torch.float32, device=dev)
        sa = torch.empty(n, dtype=torch.float32, device=dev)
        sf = torch.empty(n, dtype=torch.float32, device=dev)
        st = self.lib.covspec_score(self._ctx, C.byref(m.problem), _ptr(sq), _ptr(sa), _ptr(sf),
                                    _stream())
        if st:
            raise CovspecError(st, "covspec_score")
        return sq, (sa if self.cfg.act_layers > 0 else None), sf

    def select(self, m: _Marshalled, s_fused: torch.Tensor):
        """covspec_select: returns (keep_idx, keep_offsets, presel_idx, presel_offsets, energy)."""
        ko, po = self.plan_sizes(m)
        dev = s_fused.device
        keep_idx = torch.empty(int(ko[-1]), dtype=torch.int32, device=dev)
        presel = torch.empty(int(po[-1]), dtype=torch.int32, device=dev)
        energy = torch.empty(int(po[-1]), dtype=torch.float32, device=dev)
        ko2 = np.zeros_like(ko)
        st = self.lib.covspec_select(self._ctx, C.byref(m.problem), _ptr(s_fused), _ptr(keep_idx),
                                     ko2.ctypes.data_as(C.POINTER(C.c_int)), _ptr(presel),
                                     _ptr(energy), _stream())
        if st:
            raise CovspecError(st, "covspec_select")
        assert np.array_equal(ko, ko2)
        return keep_idx, ko, presel, po, energy

    def compact(self, m: _Marshalled, keep_idx: torch.Tensor, keep_offsets: np.ndarray):
        """covspec_compact: returns (out_hidden [sum B_vis, d], out_pos)."""
        X = m.tensors[0]
        ko, ko_p = _i32(keep_offsets)
        out = torch.empty((int(ko[-1]), X.shape[1]), dtype=X.dtype, device=X.device)
        pos = torch.empty(int(ko[-1]), dtype=torch.int32, device=X.device)
        st = self.lib.covspec_compact(self._ctx, C.byref(m.problem), _ptr(keep_idx), ko_p, _ptr(out),
                                      _ptr(pos), _stream())
        if st:
            raise CovspecError(st, "covspec_compact")
        return out, pos

    def compact_rows(self, m: _Marshalled, keep_idx: torch.Tensor, keep_offsets: np.ndarray,
                     src: torch.Tensor):
        """covspec_compact_rows: gathers the kept tokens' rows of another per-token tensor
        (first dimension = visual tokens, like X)."""
        assert src.is_cuda and src.is_contiguous() and src.shape[0] == int(m.vis[-1])
        ko, ko_p = _i32(keep_offsets)
        row_bytes = src[0].numel() * src.element_size()
        out = torch.empty((int(ko[-1]),) + tuple(src.shape[1:]), dtype=src.dtype, device=src.device)
        st = self.lib.covspec_compact_rows(self._ctx, C.byref(m.problem), _ptr(keep_idx), ko_p, _ptr(src),
                                           row_bytes, _ptr(out), _stream())
        if st:
            raise CovspecError(st, "covspec_compact_rows")
        return out

    def prune(self, m: _Marshalled, out: Optional[torch.Tensor] = None,
              keep_idx: Optional[torch.Tensor] = None):
        """covspec_prune: the fused path.  Returns (out_hidden, keep_idx, keep_offsets)."""
        X = m.tensors[0]
        ko = np.zeros(m.batch + 1, dtype=np.int32)
        if out is None or keep_idx is None:
            ko, _ = self.plan_sizes(m)
            out = torch.empty((int(ko[-1]), X.shape[1]), dtype=X.dtype, device=X.device)
            keep_idx = torch.empty(int(ko[-1]), dtype=torch.int32, device=X.device)
        st = self.lib.covspec_prune(self._ctx, C.byref(m.problem), _ptr(out), _ptr(keep_idx),
                                    ko.ctypes.data_as(C.POINTER(C.c_int)), _stream())
        if st:
            raise CovspecError(st, "covspec_prune")
        return out, keep_idx, ko

    def profile_begin(self, max_calls: int):
        st = self.lib.covspec_profile_begin(self._ctx, int(max_calls))
        if st:
            raise CovspecError(st, "covspec_profile_begin")

    def profile_end(self):
        """Returns ({stage name: summed milliseconds}, number of profiled prune calls)."""
        n = self.lib.covspec_profile_stage_count()
        ms = (C.c_double * n)()
        calls = C.c_int()
        st = self.lib.covspec_profile_end(self._ctx, ms, n, C.byref(calls))
        if st:
            raise CovspecError(st, "covspec_profile_end")
        names = [self.lib.covspec_profile_stage_name(i).decode() for i in range(n)]
        return dict(zip(names, list(ms))), calls.value

    def selftest_wait_timeout(self):
        """covspec_selftest_wait_timeout: makes one bounded wait run out on purpose."""
        st = self.lib.covspec_selftest_wait_timeout(self._ctx, _stream())
        if st:
            raise CovspecError(st, "covspec_selftest_wait_timeout")

    def iteration_counts(self, batch: int):
        """covspec_get_iteration_counts: multiplications by the Gram matrix per request of the last call."""
        out = np.zeros(batch, dtype=np.int32)
        st = self.lib.covspec_get_iteration_counts(self._ctx, int(batch), out.ctypes.data_as(C.POINTER(C.c_int)),
                                                   _stream())
        if st:
            raise CovspecError(st, "covspec_get_iteration_counts")
        return out

    def fill_workspace(self, byte: int):
        """covspec_selftest_fill_workspace: poisons the context's scratch before the next call."""
        st = self.lib.covspec_selftest_fill_workspace(self._ctx, int(byte), _stream())
        if st:
            raise CovspecError(st, "covspec_selftest_fill_workspace")

    def device_status(self) -> int:
        return int(self.lib.covspec_get_device_status(self._ctx, _stream()))

    def check_device_status(self):
        st = self.device_status()
        if st:
            raise CovspecError(st, "device status")


def _addr(t, name: str, dtype: torch.dtype, device: torch.device, least: int):
    """The address of a tensor that kernels on `device` read or write `least` elements of `dtype` from: the
    library takes addresses only, so what does not fit is refused here.  Pinned host memory is within a kernel's
    reach too.  None stays None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a tensor is required, not {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {dtype} is required, not {t.dtype}")
    if t.device != device and not (t.device.type == "cpu" and t.is_pinned()):
        raise ValueError(f"{name}: on {t.device}, the call is on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor is required")
    if t.numel() < least:
        raise ValueError(f"{name}: {t.numel()} elements, {least} are used")
    return t.data_ptr()


def _c_int(v, name: str) -> int:
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name}: {v} is no 32-bit integer")
    return v


def query_score_static(X: torch.Tensor, Q: torch.Tensor, vis_offsets, txt_offsets,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """covspec_query_score_static: Eq. 10 with the identity embedding for callers that must not
    allocate device memory (a serving loop with a fully committed memory pool, a process whose
    allocator belongs to another framework).  The library call itself allocates nothing; pass
    `out` (float32, one element per visual token) to keep this wrapper allocation-free as well."""
    if _lib is None:
        load_library()
    assert X.is_cuda and Q.is_cuda and X.is_contiguous() and Q.is_contiguous() and X.dtype == Q.dtype
    vis = np.ascontiguousarray(vis_offsets, dtype=np.int32)
    txt = np.ascontiguousarray(txt_offsets, dtype=np.int32)
    if out is None:
        out = torch.empty(int(vis[-1]), dtype=torch.float32, device=X.device)
    st = None if _native is None else _native.static_score(X, Q, vis, txt, out)
    if st is None:
        st = _static_score(X, Q, vis, txt, out)
    if st:
        raise CovspecError(st, "covspec_query_score_static")
    return out


def _static_score(X, Q, vis, txt, out) -> int:
    """The call for arguments of every kind that the library can take; says what is wrong with others."""
    if X.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"X: bfloat16 or float32 is required, not {X.dtype}")
    d = _c_int(X.shape[1], "d")
    if Q.shape[1] != d:
        raise ValueError(f"Q: {Q.shape[1]} features, X has {d}")
    if vis.size < 2 or vis.size != txt.size:
        raise ValueError(f"{vis.size} and {txt.size} offsets: one more than requests is required of both")
    rows_x, rows_q = int(vis[-1]), int(txt[-1])      # the library refuses offsets that do not ascend from 0
    ip = C.POINTER(C.c_int)
    with torch.cuda.device(X.device):
        return load_library().covspec_query_score_static(
            COVSPEC_BF16 if X.dtype == torch.bfloat16 else COVSPEC_F32, d, vis.size - 1,
            _addr(X, "X", X.dtype, X.device, rows_x * d), vis.ctypes.data_as(ip),
            _addr(Q, "Q", X.dtype, X.device, rows_q * d), txt.ctypes.data_as(ip),
            _addr(out, "out", torch.float32, X.device, rows_x), _stream())


_LOGIT_DTYPES = {torch.float32: COVSPEC_F32, torch.bfloat16: COVSPEC_BF16, torch.float16: COVSPEC_F16}


def correct(z_draft: torch.Tensor, z_target: torch.Tensor, uniforms: torch.Tensor, gamma: float,
            drafted: Optional[torch.Tensor] = None, vocab: Optional[int] = None):
    """covspec_correct: gating (Eq. 16-17), acceptance probability (Eq. 5) and the residual
    correction draw (Eq. 6) for every row of two logit matrices [rows, ld] (ld >= vocab).
    Returns (margin, gate, accept, resid_mass, token) device tensors."""
    if _lib is None:
        load_library()
    # native: on a drafted block of a few positions the call would take longer in Python than on the device
    got = None if _native is None else _native.correct(z_draft, z_target, uniforms, gamma, drafted, vocab)
    if type(got) is tuple:
        return got
    if got is not None:
        raise CovspecError(got, "covspec_correct")
    return _correct(z_draft, z_target, uniforms, gamma, drafted, vocab)


def _correct(z_draft, z_target, uniforms, gamma, drafted, vocab):
    """The call for arguments of every kind that the library can take; says what is wrong with others."""
    assert z_draft.is_cuda and z_draft.is_contiguous() and z_target.is_contiguous()
    assert z_draft.shape == z_target.shape and z_draft.dtype == z_target.dtype
    rows, ld = z_draft.shape
    dtype, dev = _LOGIT_DTYPES[z_draft.dtype], z_draft.device
    vocab = ld if vocab is None else _c_int(vocab, "vocab")
    zt = _addr(z_target, "z_target", z_draft.dtype, dev, z_draft.numel())
    y, u = _addr(drafted, "drafted", torch.int32, dev, rows), _addr(uniforms, "uniforms", torch.float32, dev, rows)
    margin, accept, mass = (torch.empty(rows, dtype=torch.float32, device=dev) for _ in range(3))
    gate, token = (torch.empty(rows, dtype=torch.int32, device=dev) for _ in range(2))
    with torch.cuda.device(dev):
        st = load_library().covspec_correct(dtype, _c_int(rows, "rows"), vocab, ld, z_draft.data_ptr(), zt, y, u, gamma,
                                            margin.data_ptr(), gate.data_ptr(), accept.data_ptr(), mass.data_ptr(),
                                            token.data_ptr(), _stream())
    if st:
        raise CovspecError(st, "covspec_correct")
    return margin, gate, accept, mass, token


def fanout(f0: int, rho: float, j: int) -> int:
    """covspec_fanout: F_j = ceil(F_0 * rho^j) (Eq. 23)."""
    v = load_library().covspec_fanout(int(f0), float(rho), int(j))
    if v < 0:
        raise CovspecError(v, "covspec_fanout")
    return v


def branch_candidates(z_draft: torch.Tensor, fanouts, drafted: Optional[torch.Tensor] = None,
                      vocab: Optional[int] = None):
    """covspec_branch_candidates: the F_j largest draft logits of every row, the drafted token
    excluded.  `fanouts`: one int per row.  Returns (cand int32 device tensor, offsets numpy)."""
    lib = _lib or load_library()
    rows, ld = z_draft.shape
    off = np.empty(rows + 1, dtype=np.int32)
    got = None if _native is None else _native.candidates(z_draft, fanouts, off, drafted, vocab)
    if isinstance(got, torch.Tensor):
        return got, off
    # fan-outs that are no list of ints, and the fan-outs and row lengths that the host-offset form does not take (-3)
    if not z_draft.is_cuda:
        raise ValueError(f"z_draft: on {z_draft.device}, a CUDA device is required")
    dtype, dev = _LOGIT_DTYPES[z_draft.dtype], z_draft.device
    z = _addr(z_draft, "z_draft", z_draft.dtype, dev, 0)
    y = _addr(drafted, "drafted", torch.int32, dev, rows)
    vocab = ld if vocab is None else _c_int(vocab, "vocab")
    f = np.asarray(fanouts, dtype=np.int64)
    assert len(f) == rows
    off = np.zeros(rows + 1, dtype=np.int32)
    np.cumsum(f, out=off[1:])
    total, most = int(off[-1]), int(f.max()) if rows else 0
    cand = torch.empty(max(total, 1), dtype=torch.int32, device=dev)
    with torch.cuda.device(dev):
        args = (dtype, _c_int(rows, "rows"), vocab, ld, z, y)
        st = lib.covspec_branch_candidates_host(*args, off.ctypes.data, most, cand.data_ptr(), _stream())
        if st == -3:
            d_off = torch.from_numpy(off).to(dev)
            st = lib.covspec_branch_candidates(*args, d_off.data_ptr(), most, cand.data_ptr(), _stream())
    if st:
        raise CovspecError(st, "covspec_branch_candidates")
    return (cand if total else cand[:0]), off


_STORES = {torch.float32: COVSPEC_F32, torch.bfloat16: COVSPEC_BF16, torch.float16: COVSPEC_F16,
           torch.float8_e4m3fn: COVSPEC_E4M3, torch.int8: COVSPEC_INT8}


def _rows(t: torch.Tensor, name: str, dtype: torch.dtype, device: torch.device, heads: int, head_dim: int):
    """(address, stride) of rows [n, heads, head_dim] that are dense but for the step from row to row."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a tensor is required, not {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {dtype} is required, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, the call is on {device}")
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != head_dim:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, [tokens, {heads}, {head_dim}] is required")
    if t.shape[0] and not t[0].is_contiguous():
        raise ValueError(f"{name}: rows have to be dense")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else heads * head_dim


class PagedCache:
    """Keys and values of one layer in pages (covspec_cache): `k`, `v` [pages, heads, page_size, head_dim] in float32,
    bfloat16, float16, float8_e4m3fn or int8, each page dense; the two 8-bit types come with `k_scale`, `v_scale` [pages, heads,
    page_size] float32.  The tensors stay the caller's: `k` and `v` may be views of one allocation.  A float32 cache is written
    and read only.  Results carry no gradient.

    The calls take the tokens of a batch, packed request by request: `offsets` [batch + 1], `lengths` [batch] and `table` [batch,
    pages of a request], int32 on the cache's device.  Request b's tokens offsets[b] .. offsets[b+1] are the last ones of its
    lengths[b] positions."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        if not (isinstance(k, torch.Tensor) and isinstance(v, torch.Tensor)) or k.dtype not in _STORES or v.dtype != k.dtype:
            raise TypeError("k, v: tensors of one type are required, float32, bfloat16, float16, float8_e4m3fn or int8")
        if not k.is_cuda or v.device != k.device:
            raise ValueError(f"k on {k.device}, v on {v.device}: one CUDA device is required")
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)}: [pages, heads, page_size, head_dim] is required of both")
        for name, t in (("k", k), ("v", v)):
            if not t.numel() or not t[0].is_contiguous():
                raise ValueError(f"{name}: dense pages are required")
        store, page = _STORES[k.dtype], k[0].numel()
        scales = (k_scale, v_scale)
        if (store >= COVSPEC_E4M3) != all(s is not None for s in scales) or (store < COVSPEC_E4M3 and any(s is not None for s in scales)):
            raise ValueError("k_scale, v_scale: required of the 8-bit types and of no other")
        pages, heads, page_size, head_dim = k.shape
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self._held = (k, v, k_scale, v_scale)      # the addresses below are theirs
        self._c = Cache(store, _c_int(pages, "pages"), _c_int(heads, "heads"), _c_int(page_size, "page_size"), head_dim,
                        k.data_ptr(), v.data_ptr(),
                        *(_addr(s, n, torch.float32, k.device, pages * heads * page_size)
                          for n, s in (("k_scale", k_scale), ("v_scale", v_scale))),
                        *(t.stride(0) if pages > 1 else page for t in (k, v)))
        self._ref, self._at, self._work = C.byref(self._c), C.addressof(self._c), {}

    @classmethod
    def empty(cls, pages: int, heads: int, page_size: int, head_dim: int, dtype: torch.dtype, device="cuda") -> "PagedCache":
        """A cache in memory of its own; what it holds is undefined until it is written."""
        k, v = (torch.empty(pages, heads, page_size, head_dim, dtype=dtype, device=device) for _ in range(2))
        if _STORES.get(dtype, -1) < COVSPEC_E4M3:
            return cls(k, v)
        return cls(k, v, *(torch.empty(pages, heads, page_size, dtype=torch.float32, device=device) for _ in range(2)))

    def _tokens(self, offsets, lengths, table) -> Tokens:
        dev = self.k.device
        for name, t, dims in (("offsets", offsets, 1), ("lengths", lengths, 1), ("table", table, 2)):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}: a tensor is required, not {type(t).__name__}")
            if t.dim() != dims:
                raise ValueError(f"{name}: {dims} dimensions are required")
        batch = lengths.shape[0]
        if table.shape[0] < batch or table.stride(1) != 1 or (batch > 1 and table.stride(0) < table.shape[1]):
            raise ValueError(f"table: rows of page ids of {batch} requests are required")
        if table.dtype != torch.int32:
            raise TypeError(f"table: {torch.int32} is required, not {table.dtype}")
        if table.device != dev:
            raise ValueError(f"table: on {table.device}, the call is on {dev}")
        return Tokens(_c_int(batch, "batch"), _addr(offsets, "offsets", torch.int32, dev, batch + 1),
                      _addr(lengths, "lengths", torch.int32, dev, batch), table.data_ptr(), _c_int(table.shape[1], "table"),
                      max(table.stride(0), table.shape[1]))

    def write(self, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor,
              rows: Optional[torch.Tensor] = None, row_offsets: Optional[torch.Tensor] = None) -> None:
        """covspec_cache_write: keys and values [tokens, heads, head_dim] (float32, bfloat16 or float16; rows may be columns of
        one projection) into the cache.  With `rows` and `row_offsets` token i of request b is row row_offsets[b] + rows[i]:
        Pruner.select's keep_idx and the visual offsets (int32, on the device) write the kept tokens of a prefill."""
        lib, dev = _lib or load_library(), self.k.device
        st = None if _native is None else _native.cache_write(self._at, self.k, k, v, offsets, lengths, table, rows, row_offsets)
        if st is None:
            st = self._write(lib, dev, k, v, offsets, lengths, table, rows, row_offsets)
        if st:
            raise CovspecError(st, "covspec_cache_write")

    def _write(self, lib, dev, k, v, offsets, lengths, table, rows, row_offsets) -> int:
        """The call for arguments of every kind that the library can take; says what is wrong with others."""
        dtype = k.dtype if isinstance(k, torch.Tensor) else None
        if dtype not in _LOGIT_DTYPES:
            raise TypeError(f"k: float32, bfloat16 or float16 is required, not {dtype}")
        heads, dim = self._c.heads, self._c.head_dim
        kp, ks = _rows(k, "k", dtype, dev, heads, dim)
        vp, vs = _rows(v, "v", dtype, dev, heads, dim)
        if k.shape[0] != v.shape[0]:
            raise ValueError(f"k, v: {k.shape[0]} and {v.shape[0]} tokens")
        tokens = self._tokens(offsets, lengths, table)
        if (rows is None) != (row_offsets is None):
            raise ValueError("rows, row_offsets: both or neither")
        n = k.shape[0] if rows is None else rows.numel()
        rp, rop = _addr(rows, "rows", torch.int32, dev, n), _addr(row_offsets, "row_offsets", torch.int32, dev, tokens.batch + 1)
        with torch.cuda.device(dev):
            return lib.covspec_cache_write(self._ref, C.byref(tokens), _LOGIT_DTYPES[dtype], _c_int(n, "tokens"), kp, vp, ks, vs, rp, rop,
                                           _c_int(k.shape[0], "rows of k"), _stream())

    def read(self, offsets: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, n: int, dtype: torch.dtype = torch.bfloat16):
        """covspec_cache_read: (k, v), [n, heads, head_dim] each, of the `n` tokens that `offsets` delimits; rows of no request
        are undefined."""
        lib, dev = _lib or load_library(), self.k.device
        if _native is not None and dtype in _LOGIT_DTYPES:
            got = _native.cache_read(self._at, self.k, offsets, lengths, table, n, _LOGIT_DTYPES[dtype])
            if type(got) is tuple:
                return got
            if got is not None:
                raise CovspecError(got, "covspec_cache_read")
        tokens = self._tokens(offsets, lengths, table)
        if dtype not in _LOGIT_DTYPES:
            raise TypeError(f"dtype: float32, bfloat16 or float16 is required, not {dtype}")
        k, v = (torch.empty(n, self._c.heads, self._c.head_dim, dtype=dtype, device=dev) for _ in range(2))
        with torch.cuda.device(dev):
            st = lib.covspec_cache_read(self._ref, C.byref(tokens), _LOGIT_DTYPES[dtype], _c_int(n, "n"), k.data_ptr(), v.data_ptr(),
                                        _stream())
        if st:
            raise CovspecError(st, "covspec_cache_read")
        return k, v

    def attend(self, q: torch.Tensor, offsets: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor,
               scale: Optional[float] = None, window: int = 0, max_new: int = 0, lse: bool = False,
               out: Optional[torch.Tensor] = None):
        """covspec_cache_attend: attention of the tokens' queries [tokens, q_heads, head_dim] (bfloat16 or float16) over the
        cache, which already holds their keys and values.  `scale`: 1 / sqrt(head_dim) if None; `window`: positions a token
        sees, itself among them, 0 for all; `max_new`: most tokens of a request, where the caller knows it (a hint).  Returns
        the rows (in `out` if given), with `lse` also the float32 log-sums [tokens, q_heads].  Rows of no request are undefined,
        in a given `out` they are left as they were."""
        lib, dev = _lib or load_library(), self.k.device
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise ValueError("q: [tokens, q_heads, head_dim] is required")
        if scale is None:
            scale = self._c.head_dim ** -0.5
        heads = q.shape[1]
        size = self._work.get(heads)
        if size is None:
            with torch.cuda.device(dev):
                size = lib.covspec_cache_attend_workspace(self._ref, _c_int(heads, "q_heads"))
            if size < 0:
                raise CovspecError(int(size), "covspec_cache_attend")
            self._work[heads] = size
        if _native is not None:
            got = _native.cache_attend(self._at, self.k, size, q, offsets, lengths, table, scale, window, max_new, lse, out)
            if got is not None:
                if type(got) is int:
                    raise CovspecError(got, "covspec_cache_attend")
                return got
        return self._attend(lib, dev, size, q, offsets, lengths, table, scale, window, max_new, lse, out)

    def _attend(self, lib, dev, size, q, offsets, lengths, table, scale, window, max_new, lse, out):
        """The call for arguments of every kind that the library can take; says what is wrong with others."""
        dtype = q.dtype
        if dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"q: bfloat16 or float16 is required, not {dtype}")
        n, heads = q.shape[0], q.shape[1]
        qp, qs = _rows(q, "q", dtype, dev, heads, self._c.head_dim)
        tokens = self._tokens(offsets, lengths, table)
        if out is None:
            out = torch.empty(n, heads, self._c.head_dim, dtype=dtype, device=dev)
        op, os_ = _rows(out, "out", dtype, dev, heads, self._c.head_dim)
        if out.shape[0] < n:
            raise ValueError(f"out: {out.shape[0]} rows, {n} are written")
        logs = torch.empty(n, heads, dtype=torch.float32, device=dev) if lse else None
        with torch.cuda.device(dev):
            # from torch's pool, like the outputs: it knows streams and captures, so no two calls in flight share it
            work = torch.empty(size, dtype=torch.uint8, device=dev)
            st = lib.covspec_cache_attend(self._ref, C.byref(tokens), _LOGIT_DTYPES[dtype], _c_int(n, "tokens"), qp, qs, heads,
                                          float(scale), _c_int(window, "window"),
                                          _c_int(max_new, "max_new"), op, os_, _ptr(logs), work.data_ptr(), size, _stream())
        if st:
            raise CovspecError(st, "covspec_cache_attend")
        return (out, logs) if lse else out


def edit_logits(z: torch.Tensor, row_offsets: torch.Tensor, *, history: Optional[torch.Tensor] = None,
                history_offsets: Optional[torch.Tensor] = None, prompt_lengths: Optional[torch.Tensor] = None,
                drafted: Optional[torch.Tensor] = None, repetition: Optional[torch.Tensor] = None,
                presence: Optional[torch.Tensor] = None, frequency: Optional[torch.Tensor] = None,
                bias_ids: Optional[torch.Tensor] = None, bias_values: Optional[torch.Tensor] = None,
                bias_offsets: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                vocab: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """covspec_edit_logits: repetition, frequency and presence penalties, biases and a grammar's mask on the logits [rows, ld] of
    drafted blocks, before `correct` or `branch_candidates`.  `row_offsets` [batch + 1] delimits the requests' rows; row j of a
    request counts the tokens `drafted` at its rows before j as history.  `mask`: int32 [rows, ceil(vocab / 32)], bit w % 32 of
    word w / 32 allows token w.  Everything on z's device, ids and offsets int32, factors float32.  Returns the edited logits (in
    `out` if given, which may be z), without a gradient; rows of no request and columns past the vocabulary are undefined, or left as
    they were."""
    lib = _lib or load_library()
    if _native is not None:
        got = _native.edit_logits(z, row_offsets, history, history_offsets, prompt_lengths, drafted, repetition, presence, frequency,
                                  bias_ids, bias_values, bias_offsets, mask, vocab, out)
        if got is not None:
            if type(got) is int:
                raise CovspecError(got, "covspec_edit_logits")
            return got
    if not isinstance(z, torch.Tensor) or z.dim() != 2 or z.dtype not in _LOGIT_DTYPES:
        raise TypeError("z: a matrix of float32, bfloat16 or float16 is required")
    if not z.is_cuda:
        raise ValueError(f"z: on {z.device}, a CUDA device is required")
    rows, ld = z.shape
    dev = z.device
    zp = _addr(z, "z", z.dtype, dev, 0)
    vocab = ld if vocab is None else _c_int(vocab, "vocab")
    if out is None:
        out = torch.empty_like(z)
    elif isinstance(out, torch.Tensor) and out.shape != z.shape:
        raise ValueError(f"out: shape {tuple(out.shape)}, z has {tuple(z.shape)}")
    if not isinstance(row_offsets, torch.Tensor) or row_offsets.numel() < 2:
        raise ValueError("row_offsets: a tensor of one more than requests is required")
    batch, i32, f32 = row_offsets.numel() - 1, torch.int32, torch.float32
    if (history is None) != (history_offsets is None):
        raise ValueError("history, history_offsets: both or neither")
    if len({bias_ids is None, bias_values is None, bias_offsets is None}) > 1:
        raise ValueError("bias_ids, bias_values, bias_offsets: all or none")
    n_hist, n_bias = 0 if history is None else history.numel(), 0 if bias_ids is None else bias_ids.numel()
    e = Edits(_c_int(batch, "batch"), _addr(row_offsets, "row_offsets", i32, dev, batch + 1), _addr(history, "history", i32, dev, 0),
              _addr(history_offsets, "history_offsets", i32, dev, batch + 1), _c_int(n_hist, "history"),
              _addr(prompt_lengths, "prompt_lengths", i32, dev, batch), _addr(drafted, "drafted", i32, dev, rows),
              _addr(repetition, "repetition", f32, dev, batch), _addr(presence, "presence", f32, dev, batch),
              _addr(frequency, "frequency", f32, dev, batch), _addr(bias_ids, "bias_ids", i32, dev, 0),
              _addr(bias_values, "bias_values", f32, dev, n_bias), _addr(bias_offsets, "bias_offsets", i32, dev, batch + 1),
              _c_int(n_bias, "bias_ids"))
    if mask is not None:
        words = (vocab + 31) // 32
        if not isinstance(mask, torch.Tensor) or mask.dim() != 2 or mask.shape[0] < rows or mask.shape[1] < words:
            raise ValueError(f"mask: at least [{rows}, {words}] is required")
        e.mask, e.mask_stride = _addr(mask, "mask", i32, dev, rows * words), 4 * mask.shape[1]
    op = _addr(out, "out", z.dtype, dev, z.numel())
    with torch.cuda.device(dev):
        st = lib.covspec_edit_logits(_LOGIT_DTYPES[z.dtype], _c_int(rows, "rows"), vocab, ld, zp, op, C.byref(e), _stream())
    if st:
        raise CovspecError(st, "covspec_edit_logits")
    return out
