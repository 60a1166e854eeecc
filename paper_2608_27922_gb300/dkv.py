"""Thin ctypes binding of libdkv.so (include/dkv.h), with the same names as the C ABI.

Only argument marshalling happens here: torch tensors are checked for device,
dtype, shape and contiguity and passed as raw device pointers; every step of
the bank update and of attention runs in the CUDA library.  There is no CPU or
PyTorch fallback: if the library cannot be loaded, ``lib()`` raises.

``BankLayer`` is a convenience owner of one layer's caller-owned buffers
(bank tensors and workspace, allocated with torch) around a ``dkv_bank_t``.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "lib", "libdkv.so")

DKV_OK = 0
DKV_DTYPE_BF16, DKV_DTYPE_FP32 = 0, 1
DKV_SCORE_TENSOR, DKV_SCORE_FP32 = 0, 1
DKV_ORDER_SCORE, DKV_ORDER_SOURCE = 0, 1
DKV_DESC_K, DKV_DESC_KV = 0, 1
DKV_EVICT_MANDATORY_DENSEST, DKV_EVICT_DENSEST, DKV_EVICT_MANDATORY_SOURCE = 0, 1, 2
STATUS = {0: "DKV_OK", 1: "DKV_ERR_ARG", 2: "DKV_ERR_SHAPE", 3: "DKV_ERR_STATE", 4: "DKV_ERR_CUDA",
          5: "DKV_ERR_NOMEM", 6: "DKV_ERR_TIMEOUT", 7: "DKV_ERR_UNSUPPORTED", 8: "DKV_ERR_DEVICE"}


class dkv_params_t(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("sigma", ctypes.c_float), ("p", ctypes.c_float),
                ("eps", ctypes.c_float), ("delta", ctypes.c_float), ("sync_heads", ctypes.c_int32),
                ("score_mode", ctypes.c_int32), ("order", ctypes.c_int32), ("eviction", ctypes.c_int32),
                ("refresh_baselines", ctypes.c_int32), ("layer_heads", ctypes.c_int32),
                ("descriptor", ctypes.c_int32)]


class dkv_buffers_t(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("rho", ctypes.c_void_p),
                ("base", ctypes.c_void_p), ("knorm", ctypes.c_void_p), ("prov_step", ctypes.c_void_p),
                ("prov_src", ctypes.c_void_p), ("occupancy", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class dkv_layer_stats_t(ctypes.Structure):
    _fields_ = [("r_star", ctypes.c_int32), ("rmax", ctypes.c_int32), ("n_candidates", ctypes.c_int32),
                ("empty_init", ctypes.c_int32)]


class dkv_head_stats_t(ctypes.Structure):
    _fields_ = [("occupancy_before", ctypes.c_int32), ("occupancy_after", ctypes.c_int32),
                ("admitted", ctypes.c_int32), ("evicted", ctypes.c_int32), ("mandatory", ctypes.c_int32),
                ("pre_violators", ctypes.c_int32)]


class dkv_intermediates_t(ctypes.Structure):
    _fields_ = [("score", ctypes.c_void_p), ("perm", ctypes.c_void_p), ("cross", ctypes.c_void_p),
                ("rho_tilde", ctypes.c_void_p), ("slot_new", ctypes.c_void_p), ("n_max", ctypes.c_int64),
                ("M_max", ctypes.c_int64)]


class dkv_cache_buffers_t(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class dkv_cache_seqs_t(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("seq_len", ctypes.c_void_p), ("row_start", ctypes.c_void_p),
                ("n_seq", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


class dkv_cache_attend_t(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("block", ctypes.c_int32), ("max_rows", ctypes.c_int32)]


class dkv_norm_rope_t(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_void_p), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("norm", ctypes.c_int32), ("layout", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("axis_pairs", ctypes.c_int32 * 4)]


class dkv_cache_table_t(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("seq_len", ctypes.c_void_p), ("n_seq", ctypes.c_int32),
                ("max_pages", ctypes.c_int32)]


class dkv_cache_summaries_t(ctypes.Structure):
    _fields_ = [("code", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class dkv_cache_choose_t(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int32), ("block", ctypes.c_int32), ("sink_pages", ctypes.c_int32),
                ("local_pages", ctypes.c_int32), ("top", ctypes.c_int32), ("width", ctypes.c_int32)]


class dkv_cache_chosen_t(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("tile", ctypes.c_int32), ("block", ctypes.c_int32), ("width", ctypes.c_int32)]


# (name, restype, argtypes) of every exported symbol declared in include/dkv.h
_P = ctypes.c_void_p
_I = ctypes.c_int32
_L = ctypes.c_int64
SIGNATURES = [
    ("dkv_status_str", ctypes.c_char_p, [_I]),
    ("dkv_version", _I, []),
    ("dkv_params_default", _I, [ctypes.POINTER(dkv_params_t), _I]),
    ("dkv_bank_workspace_size", ctypes.c_size_t, [_I, _I, ctypes.POINTER(ctypes.c_int32), _I, _I]),
    ("dkv_bank_workspace_size_ex", ctypes.c_size_t, [_I, _I, ctypes.POINTER(ctypes.c_int32), _I, _I,
                                                     ctypes.POINTER(dkv_params_t)]),
    ("dkv_bank_create", _I, [ctypes.POINTER(_P), _I, _I, ctypes.POINTER(ctypes.c_int32), _I, _I,
                             ctypes.POINTER(dkv_params_t), ctypes.POINTER(dkv_buffers_t)]),
    ("dkv_bank_destroy", None, [_P]),
    ("dkv_bank_reset", _I, [_P, _P]),
    ("dkv_bank_admit", _I, [_P, _P, _P, _I, ctypes.c_int64, _P]),
    ("dkv_bank_admit_rope", _I, [_P, _P, _P, _I, ctypes.c_int64, _P, _P, _I, _P]),
    ("dkv_bank_compress", _I, [_P, _P]),
    ("dkv_bank_evict", _I, [_P, _P]),
    ("dkv_bank_commit", _I, [_P, _P]),
    ("dkv_bank_attend", _I, [_P, _P, _I, _P, _P, _I, _P, _P]),
    ("dkv_bank_import", _I, [_P, ctypes.POINTER(ctypes.c_int32), _P]),
    ("dkv_bank_export", _I, [_P, ctypes.POINTER(dkv_buffers_t)]),
    ("dkv_bank_sync", _I, [_P]),
    ("dkv_bank_stats", _I, [_P, ctypes.POINTER(dkv_layer_stats_t), ctypes.POINTER(dkv_head_stats_t)]),
    ("dkv_bank_occupancy", _I, [_P, ctypes.POINTER(ctypes.c_int32)]),
    ("dkv_bank_intermediates", _I, [_P, ctypes.POINTER(dkv_intermediates_t)]),
    ("dkv_bank_set_timing", _I, [_P, _I]),
    ("dkv_bank_kernel_times", _I, [_P, _I, ctypes.c_char_p, ctypes.POINTER(ctypes.c_int32),
                                   ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)]),
    ("dkv_candidate_order_noalloc", _I, [_P, _P, _I, _P, _I, _I, _I, ctypes.POINTER(dkv_params_t), _P, _P, _P]),
    ("dkv_selftest_wait_timeout", _I, [_I, ctypes.POINTER(ctypes.c_int64)]),
    ("dkv_sequential_scratch_size", ctypes.c_size_t, [_I, _I, _I, _I]),
    ("dkv_bank_update_sequential", _I, [_P, _P, _P, _I, ctypes.c_int64, _P, ctypes.c_size_t, _P]),
    ("dkv_cache_create", _I, [ctypes.POINTER(_P), _I, _I, _I, _I, _I, ctypes.POINTER(dkv_cache_buffers_t)]),
    ("dkv_cache_destroy", None, [_P]),
    ("dkv_cache_write", _I, [_P, ctypes.POINTER(dkv_cache_seqs_t), _P, _P, _I, _L, _L, _L, _L, _P]),
    ("dkv_cache_read", _I, [_P, ctypes.POINTER(dkv_cache_seqs_t), _P, _P, _P, _I, _L, _L, _L, _L, _P]),
    ("dkv_cache_attend_scratch_size", ctypes.c_size_t, [_P, _I, _I, _I, _I]),
    ("dkv_cache_attend", _I, [_P, ctypes.POINTER(dkv_cache_seqs_t), _P, _I, _I, _L, _L, _P, _L, _L,
                              ctypes.POINTER(dkv_cache_attend_t), _P, ctypes.c_size_t, _P]),
    ("dkv_cache_sync", _I, [_P]),
    ("dkv_norm_rope", _I, [_I, ctypes.POINTER(dkv_norm_rope_t), _P, _I, _I, _P, _L, _L, _P, _L, _L, _I, _P, _L, _L, _P, _L, _L,
                           _P]),
    ("dkv_cache_write_norm_rope", _I, [_P, ctypes.POINTER(dkv_cache_seqs_t), ctypes.POINTER(dkv_norm_rope_t), _P, _I, _I, _P, _L,
                                       _L, _P, _L, _L, _P, _L, _L, _P, _L, _L, _P]),
    ("dkv_cache_fork", _I, [_P, _P, ctypes.POINTER(dkv_cache_table_t), _P, ctypes.POINTER(dkv_cache_table_t), _P]),
    ("dkv_cache_extend_scratch_size", ctypes.c_size_t, [_P, _I]),
    ("dkv_cache_extend", _I, [_P, _P, ctypes.POINTER(dkv_cache_table_t), _P, _P, ctypes.c_size_t, _P]),
    ("dkv_cache_release", _I, [_P, _P, ctypes.POINTER(dkv_cache_table_t), _P, _P, _P]),
    ("dkv_cache_compact_scratch_size", ctypes.c_size_t, [_P, _I]),
    ("dkv_cache_compact", _I, [_P, _P, ctypes.POINTER(dkv_cache_table_t), _P, _I, _P, ctypes.POINTER(dkv_cache_table_t), _P,
                               ctypes.c_size_t, _P]),
    ("dkv_cache_summarise", _I, [_P, ctypes.POINTER(dkv_cache_seqs_t), _P, ctypes.POINTER(dkv_cache_summaries_t), _P]),
    ("dkv_cache_choose", _I, [_P, ctypes.POINTER(dkv_cache_seqs_t), ctypes.POINTER(dkv_cache_summaries_t), _P, _I, _I, _L, _L,
                              ctypes.POINTER(dkv_cache_choose_t), _P, _P]),
    ("dkv_cache_attend_chosen", _I, [_P, ctypes.POINTER(dkv_cache_seqs_t), _P, _I, _I, _L, _L, _P, _L, _L, _P,
                                     ctypes.POINTER(dkv_cache_chosen_t), _P]),
]

DKV_NOALLOC_MAX_N = 16384

_LIB: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """Loads libdkv.so (built in-tree by ``build.py``); raises if it is missing."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2608_27922_gb300.build.build()")
        L = ctypes.CDLL(LIB_PATH)
        for name, res, args in SIGNATURES:
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _LIB = L
    return _LIB


class DkvError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {STATUS.get(status, status)} ({lib().dkv_status_str(status).decode()})")


def _check(status: int, what: str) -> None:
    if status != DKV_OK:
        raise DkvError(status, what)


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ptr(t) -> int:
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    return t.data_ptr()


def _i32(xs: Sequence[int]):
    return (ctypes.c_int32 * len(xs))(*[int(x) for x in xs])


# ----------------------------------------------------------------- C ABI, same names
def dkv_version() -> int:
    return lib().dkv_version()


def dkv_params_default(d: int) -> dkv_params_t:
    p = dkv_params_t()
    _check(lib().dkv_params_default(ctypes.byref(p), d), "dkv_params_default")
    return p


def dkv_bank_workspace_size(H: int, d: int, budgets: Sequence[int], n_max: int, dtype: int,
                            params: Optional[dkv_params_t] = None) -> int:
    if params is None:
        return int(lib().dkv_bank_workspace_size(H, d, _i32(budgets), n_max, dtype))
    return int(lib().dkv_bank_workspace_size_ex(H, d, _i32(budgets), n_max, dtype, ctypes.byref(params)))


def dkv_bank_create(H: int, d: int, budgets: Sequence[int], n_max: int, dtype: int, params: dkv_params_t,
                    buffers: dkv_buffers_t) -> int:
    h = ctypes.c_void_p()
    _check(lib().dkv_bank_create(ctypes.byref(h), H, d, _i32(budgets), n_max, dtype, ctypes.byref(params),
                                 ctypes.byref(buffers)), "dkv_bank_create")
    return h.value


def dkv_bank_destroy(bank: int) -> None:
    lib().dkv_bank_destroy(bank)


def dkv_bank_reset(bank: int, stream=None) -> None:
    _check(lib().dkv_bank_reset(bank, _stream(stream)), "dkv_bank_reset")


def dkv_bank_admit(bank: int, Kc, Vc, N: int, step: int, stream=None) -> None:
    _check(lib().dkv_bank_admit(bank, _ptr(Kc), _ptr(Vc), N, step, _stream(stream)), "dkv_bank_admit")


DKV_ROPE_INTERLEAVED, DKV_ROPE_HALF = 0, 1


def dkv_bank_admit_rope(bank: int, Kc, Vc, N: int, step: int, t_coord, theta, layout: int, stream=None) -> None:
    _check(lib().dkv_bank_admit_rope(bank, _ptr(Kc), _ptr(Vc), N, step, _ptr(t_coord), _ptr(theta), layout,
                                     _stream(stream)), "dkv_bank_admit_rope")


def dkv_sequential_scratch_size(H: int, d: int, n_max: int, dtype: int) -> int:
    return int(lib().dkv_sequential_scratch_size(H, d, n_max, dtype))


def dkv_bank_update_sequential(bank: int, Kc, Vc, N: int, step: int, scratch, scratch_bytes: int,
                               stream=None) -> None:
    _check(lib().dkv_bank_update_sequential(bank, _ptr(Kc), _ptr(Vc), N, step, _ptr(scratch), scratch_bytes,
                                            _stream(stream)), "dkv_bank_update_sequential")


def dkv_bank_compress(bank: int, stream=None) -> None:
    _check(lib().dkv_bank_compress(bank, _stream(stream)), "dkv_bank_compress")


def dkv_bank_evict(bank: int, stream=None) -> None:
    _check(lib().dkv_bank_evict(bank, _stream(stream)), "dkv_bank_evict")


def dkv_bank_commit(bank: int, stream=None) -> None:
    _check(lib().dkv_bank_commit(bank, _stream(stream)), "dkv_bank_commit")


def dkv_bank_attend(bank: int, Q, Nq: int, Kw, Vw, W: int, O, stream=None) -> None:
    _check(lib().dkv_bank_attend(bank, _ptr(Q), Nq, _ptr(Kw), _ptr(Vw), W, _ptr(O), _stream(stream)),
           "dkv_bank_attend")


def dkv_bank_import(bank: int, occupancy: Sequence[int], stream=None) -> None:
    _check(lib().dkv_bank_import(bank, _i32(occupancy), _stream(stream)), "dkv_bank_import")


def dkv_bank_export(bank: int, dst: dkv_buffers_t) -> None:
    _check(lib().dkv_bank_export(bank, ctypes.byref(dst)), "dkv_bank_export")


def dkv_bank_sync(bank: int) -> None:
    _check(lib().dkv_bank_sync(bank), "dkv_bank_sync")


def dkv_bank_stats(bank: int, H: int, n_layers: int = 1) -> Tuple[List[dkv_layer_stats_t], List[dkv_head_stats_t]]:
    Ls = (dkv_layer_stats_t * n_layers)()
    arr = (dkv_head_stats_t * H)()
    _check(lib().dkv_bank_stats(bank, Ls, arr), "dkv_bank_stats")
    return list(Ls), list(arr)


def dkv_bank_occupancy(bank: int, H: int) -> List[int]:
    arr = (ctypes.c_int32 * H)()
    _check(lib().dkv_bank_occupancy(bank, arr), "dkv_bank_occupancy")
    return list(arr)


def dkv_bank_intermediates(bank: int) -> dkv_intermediates_t:
    x = dkv_intermediates_t()
    _check(lib().dkv_bank_intermediates(bank, ctypes.byref(x)), "dkv_bank_intermediates")
    return x


def dkv_bank_set_timing(bank: int, enable) -> None:
    """enable: False/0 off, True/1 every kernel, 2 attention launches only (others counted)."""
    _check(lib().dkv_bank_set_timing(bank, int(enable)), "dkv_bank_set_timing")


def dkv_bank_kernel_times(bank: int) -> Dict[str, Tuple[int, float]]:
    n = ctypes.c_int32()
    _check(lib().dkv_bank_kernel_times(bank, 0, None, None, None, ctypes.byref(n)), "dkv_bank_kernel_times")
    k = n.value
    names = ctypes.create_string_buffer(48 * max(k, 1))
    launches = (ctypes.c_int32 * max(k, 1))()
    ms = (ctypes.c_double * max(k, 1))()
    _check(lib().dkv_bank_kernel_times(bank, k, names, launches, ms, ctypes.byref(n)), "dkv_bank_kernel_times")
    out = {}
    for i in range(min(k, n.value)):
        nm = names.raw[48 * i:48 * (i + 1)].split(b"\0", 1)[0].decode()
        out[nm] = (int(launches[i]), float(ms[i]))
    return out


def dkv_candidate_order_noalloc(K_bank, base, m: int, Kc, N: int, d: int, dtype: int, params: dkv_params_t,
                                scores_out, perm_out, stream=None) -> None:
    """Eq. 6 scores and their stable order for one head, with no device allocation
    (for callers that cannot allocate; see include/dkv.h)."""
    _check(lib().dkv_candidate_order_noalloc(_ptr(K_bank) if m > 0 else 0, _ptr(base) if m > 0 else 0, m,
                                             _ptr(Kc), N, d, dtype, ctypes.byref(params), _ptr(scores_out),
                                             _ptr(perm_out), _stream(stream)), "dkv_candidate_order_noalloc")


def dkv_selftest_wait_timeout(limit_us: int):
    """Runs the bounded-wait self-test; returns (status, elapsed_ns).  DKV_ERR_TIMEOUT (6)
    is the expected status: the wait gave up after limit_us as designed."""
    el = ctypes.c_int64(0)
    st = lib().dkv_selftest_wait_timeout(int(limit_us), ctypes.byref(el))
    return int(st), int(el.value)


# ----------------------------------------------------------------- buffer owner
_TORCH_DTYPE = {DKV_DTYPE_BF16: torch.bfloat16, DKV_DTYPE_FP32: torch.float32}


def _view(ptr: int, shape, dtype: torch.dtype, device) -> torch.Tensor:
    """Wraps a device pointer owned by the library handle as a read-only-by-convention tensor."""
    n = 1
    for s in shape:
        n *= s
    esize = torch.empty(0, dtype=dtype).element_size()

    class _Arr:
        __cuda_array_interface__ = {
            "shape": (n,), "typestr": {torch.float32: "<f4", torch.int32: "<i4"}[dtype],
            "data": (ptr, False), "version": 3, "strides": (esize,)}

    return torch.as_tensor(_Arr(), device=device).view(*shape)


class BankLayer:
    """H per-head banks (one layer, or H / layer_heads layers when the layer_heads
    parameter is set): allocates the caller-owned buffers with torch and drives the C
    ABI.  All methods enqueue on the current (or given) stream."""

    def __init__(self, H: int, d: int, budgets: Sequence[int], n_max: int, dtype: torch.dtype = torch.bfloat16,
                 params: Optional[dkv_params_t] = None, device="cuda", **param_overrides):
        self.H, self.d, self.n_max = H, d, n_max
        self.budgets = [int(b) for b in budgets]
        assert len(self.budgets) == H
        self.M_max = max(self.budgets)
        self.dtype_code = {torch.bfloat16: DKV_DTYPE_BF16, torch.float32: DKV_DTYPE_FP32}[dtype]
        self.dtype = dtype
        dev = torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        p = params if params is not None else dkv_params_default(d)
        for k, v in param_overrides.items():
            setattr(p, k, v)
        self.params = p
        self.n_layers = H // p.layer_heads if p.layer_heads > 0 else 1
        dev = self.device
        self.k = torch.zeros(H, self.M_max, d, dtype=dtype, device=dev)
        self.v = torch.zeros(H, self.M_max, d, dtype=dtype, device=dev)
        self.rho = torch.zeros(H, self.M_max, dtype=torch.float32, device=dev)
        self.base = torch.zeros(H, self.M_max, dtype=torch.float32, device=dev)
        self.knorm = torch.zeros(H, self.M_max, dtype=torch.float32, device=dev)
        self.prov_step = torch.full((H, self.M_max), -1, dtype=torch.int64, device=dev)
        self.prov_src = torch.full((H, self.M_max), -1, dtype=torch.int32, device=dev)
        self.occupancy = torch.zeros(H, dtype=torch.int32, device=dev)
        ws = dkv_bank_workspace_size(H, d, self.budgets, n_max, self.dtype_code, p)
        if ws == 0:
            raise ValueError("invalid bank shape")
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=dev)
        bufs = dkv_buffers_t(self.k.data_ptr(), self.v.data_ptr(), self.rho.data_ptr(), self.base.data_ptr(),
                             self.knorm.data_ptr(), self.prov_step.data_ptr(), self.prov_src.data_ptr(),
                             self.occupancy.data_ptr(), self.workspace.data_ptr(), ws)
        self.handle = dkv_bank_create(H, d, self.budgets, n_max, self.dtype_code, p, bufs)

    def close(self):
        if getattr(self, "handle", None):
            dkv_bank_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _chk(self, t: torch.Tensor, shape, name: str):
        if t.dtype != self.dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"{name}: expected contiguous {self.dtype} {tuple(shape)} on {self.device}, "
                             f"got {t.dtype} {tuple(t.shape)} on {t.device}")

    def reset(self, stream=None):
        dkv_bank_reset(self.handle, stream)

    def admit(self, Kc: torch.Tensor, Vc: torch.Tensor, step: int, stream=None, t_coord=None, theta=None,
              rope_layout: int = DKV_ROPE_INTERLEAVED):
        """Steps 1-2.  With t_coord (int32 [N]) and theta (fp32 [d/2]) on the device, the
        keys are first rotated back to temporal rotary coordinate 0 (dkv_bank_admit_rope)."""
        N = Kc.shape[1]
        self._chk(Kc, (self.H, N, self.d), "Kc")
        self._chk(Vc, (self.H, N, self.d), "Vc")
        if (t_coord is None) != (theta is None):
            raise ValueError("t_coord and theta go together")
        if t_coord is None:
            self._pending = (Kc, Vc)   # keep the candidates alive until commit
            dkv_bank_admit(self.handle, Kc, Vc, N, step, stream)
            return
        for x, dt, shape, name in ((t_coord, torch.int32, (N,), "t_coord"), (theta, torch.float32, (self.d // 2,), "theta")):
            if x.dtype != dt or tuple(x.shape) != shape or not x.is_contiguous() or x.device != self.device:
                raise ValueError(f"{name}: expected contiguous {dt} {shape} on {self.device}")
        self._pending = (Kc, Vc, t_coord, theta)
        dkv_bank_admit_rope(self.handle, Kc, Vc, N, step, t_coord, theta, rope_layout, stream)

    def compress(self, stream=None):
        dkv_bank_compress(self.handle, stream)

    def evict(self, stream=None):
        """First half of compress; leaves k, v and occupancy untouched."""
        dkv_bank_evict(self.handle, stream)

    def commit(self, stream=None):
        """Second half of compress; order every reader of the old bank before it."""
        dkv_bank_commit(self.handle, stream)

    def update(self, Kc: torch.Tensor, Vc: torch.Tensor, step: int, stream=None, **rope):
        self.admit(Kc, Vc, step, stream, **rope)
        self.compress(stream)

    def update_sequential(self, Kc: torch.Tensor, Vc: torch.Tensor, step: int, stream=None):
        """Within-block competition: the block's candidates offered one at a time (the
        C ABI's dkv_bank_update_sequential); synchronises once with the stream."""
        N = Kc.shape[1]
        self._chk(Kc, (self.H, N, self.d), "Kc")
        self._chk(Vc, (self.H, N, self.d), "Vc")
        if getattr(self, "_seq_scratch", None) is None:
            n = dkv_sequential_scratch_size(self.H, self.d, self.n_max, self.dtype_code)
            self._seq_scratch = torch.empty(n, dtype=torch.uint8, device=self.device)
        dkv_bank_update_sequential(self.handle, Kc, Vc, N, step, self._seq_scratch, self._seq_scratch.numel(),
                                   stream)

    def attend(self, Q: torch.Tensor, Kw: Optional[torch.Tensor], Vw: Optional[torch.Tensor],
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        Nq = Q.shape[1]
        self._chk(Q, (self.H, Nq, self.d), "Q")
        W = 0 if Kw is None else Kw.shape[1]
        if W:
            self._chk(Kw, (self.H, W, self.d), "Kw")
            self._chk(Vw, (self.H, W, self.d), "Vw")
        if out is None:
            out = torch.empty_like(Q)
        self._chk(out, (self.H, Nq, self.d), "out")
        dkv_bank_attend(self.handle, Q, Nq, Kw if W else None, Vw if W else None, W, out, stream)
        return out

    def import_state(self, occupancy: Sequence[int], stream=None):
        dkv_bank_import(self.handle, occupancy, stream)

    def export_state(self, device="cpu") -> Dict[str, torch.Tensor]:
        """Checkpoint of every head (k, v, rho, base, prov_step, prov_src, occupancy), copied
        by dkv_bank_export into new tensors on `device` (host tensors are pinned)."""
        dev = torch.device(device)
        pin = dev.type == "cpu"
        H, M, d = self.H, self.M_max, self.d

        def new(shape, dtype):
            return torch.empty(shape, dtype=dtype, device=dev, pin_memory=pin)
        out = {"k": new((H, M, d), self.dtype), "v": new((H, M, d), self.dtype),
               "rho": new((H, M), torch.float32), "base": new((H, M), torch.float32),
               "prov_step": new((H, M), torch.int64), "prov_src": new((H, M), torch.int32),
               "occupancy": new((H,), torch.int32)}
        dst = dkv_buffers_t()
        for name in ("k", "v", "rho", "base", "prov_step", "prov_src", "occupancy"):
            setattr(dst, name, out[name].data_ptr())
        dkv_bank_export(self.handle, dst)
        return out

    def sync(self):
        dkv_bank_sync(self.handle)

    def stats(self):
        """(statistics of the first layer, per-head statistics of every head)."""
        Ls, hs = dkv_bank_stats(self.handle, self.H, self.n_layers)
        return Ls[0], hs

    def layer_stats(self) -> List[dkv_layer_stats_t]:
        """Statistics of each of the handle's layers (params.layer_heads heads each)."""
        return dkv_bank_stats(self.handle, self.H, self.n_layers)[0]

    def occupancy_host(self) -> List[int]:
        return dkv_bank_occupancy(self.handle, self.H)

    def intermediates(self) -> Dict[str, torch.Tensor]:
        x = dkv_bank_intermediates(self.handle)
        H, n, M = self.H, int(x.n_max), int(x.M_max)
        return {"score": _view(x.score, (H, n), torch.float32, self.device),
                "perm": _view(x.perm, (H, n), torch.int32, self.device),
                "cross": _view(x.cross, (H, M), torch.int32, self.device),
                "rho_tilde": _view(x.rho_tilde, (H, M), torch.float32, self.device),
                "slot_new": _view(x.slot_new, (H, n), torch.int32, self.device)}

    def set_timing(self, on: bool, attention_only: bool = False):
        dkv_bank_set_timing(self.handle, 2 if (on and attention_only) else int(bool(on)))

    def kernel_times(self):
        return dkv_bank_kernel_times(self.handle)


# ----------------------------------------------------------------- paged cache of the window
DKV_CACHE_BF16, DKV_CACHE_E4M3 = 0, 1
_CACHE_FORMAT = {"bf16": DKV_CACHE_BF16, "e4m3": DKV_CACHE_E4M3}


def _raw_stream(device: int) -> int:
    """cuda_stream of the device's current stream (torch's own query, without a Stream object around it)."""
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(device) if get is not None else torch.cuda.current_stream(device).cuda_stream


class CacheSeqs:
    """The sequences of a cache call (device int32 tensors, see include/dkv.h): block_table
    [n_seq][max_pages], seq_len [n_seq], row_start [n_seq + 1].  The tensors are kept and read when
    the calls' work runs; a program updates them in place between calls."""

    def __init__(self, block_table: torch.Tensor, seq_len: torch.Tensor, row_start: torch.Tensor):
        n = seq_len.numel()
        for t, shape, name in ((block_table, (n, block_table.shape[-1]), "block_table"), (seq_len, (n,), "seq_len"),
                               (row_start, (n + 1,), "row_start")):
            if (t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous()
                    or t.device != seq_len.device or not t.is_cuda):
                raise ValueError(f"{name}: expected contiguous {torch.int32} {shape} on one CUDA device, "
                                 f"got {t.dtype} {tuple(t.shape)} on {t.device}")
        self.block_table, self.seq_len, self.row_start = block_table, seq_len, row_start
        self.n_seq, self.device = n, seq_len.device
        self._c = dkv_cache_seqs_t(block_table.data_ptr(), seq_len.data_ptr(), row_start.data_ptr(), n,
                                   block_table.shape[-1])
        self._ref = ctypes.byref(self._c)


class PageTable:
    """Pages of several sequences for the calls that change them (device int32 tensors, see include/dkv.h):
    block_table [n_seq][max_pages], seq_len [n_seq].  The tensors are kept and changed in place; a CacheSeqs on the
    same ones sees what the calls made of them."""

    def __init__(self, block_table: torch.Tensor, seq_len: torch.Tensor):
        n = seq_len.numel()
        _check_i32(block_table, (n, block_table.shape[-1]), "block_table", seq_len.device)
        _check_i32(seq_len, (n,), "seq_len", seq_len.device)
        if not seq_len.is_cuda:
            raise ValueError(f"seq_len: expected a CUDA tensor, got {seq_len.device}")
        self.block_table, self.seq_len, self.n_seq, self.device = block_table, seq_len, n, seq_len.device
        self._c = dkv_cache_table_t(block_table.data_ptr(), seq_len.data_ptr(), n, block_table.shape[-1])
        self._ref = ctypes.byref(self._c)


def _check_i32(t: torch.Tensor, shape, name: str, device) -> None:
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name}: expected contiguous {torch.int32} {shape} on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def _check_32(**values) -> None:
    for name, x in values.items():
        if not -2 ** 31 <= x < 2 ** 31:                # (ctypes would take it modulo 2^32)
            raise ValueError(f"{name}: expected a 32-bit integer, got {x}")


def _check_rows(t: torch.Tensor, heads: int, rows: int, d: int, device, name: str):
    """Strides of a packed tensor between heads and rows."""
    s = t.stride()
    if t.dtype is not torch.bfloat16 or t.shape != (heads, rows, d) or t.device != device or s[2] != 1:
        raise ValueError(f"{name}: expected {torch.bfloat16} {(heads, rows, d)} with contiguous rows on "
                         f"{device}, got {t.dtype} {tuple(t.shape)}, strides {s}, on {t.device}")
    return s


class NormRope:
    """How queries and keys are normed and rotated (dkv_norm_rope_t): theta [d / 2] fp32, the frequency of each pair;
    axis_pairs, how many pairs follow each coordinate of a token (default: one coordinate); layout DKV_ROPE_INTERLEAVED
    or DKV_ROPE_HALF; norm with q_weight and k_weight [d] fp32 (None: ones) and eps.  The tensors are kept."""

    def __init__(self, d: int, theta: torch.Tensor, axis_pairs: Optional[Sequence[int]] = None,
                 layout: int = DKV_ROPE_INTERLEAVED, norm: bool = True, eps: float = 1e-6,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None):
        pairs = [d // 2] if axis_pairs is None else [int(x) for x in axis_pairs]
        if not 1 <= len(pairs) <= 4 or min(pairs) < 0 or sum(pairs) != d // 2:
            raise ValueError(f"axis_pairs: expected 1 to 4 numbers of pairs, {d // 2} together, got {pairs}")
        for t, n, name in ((theta, d // 2, "theta"), (q_weight, d, "q_weight"), (k_weight, d, "k_weight")):
            if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (n,) or not t.is_contiguous()
                                  or t.device != theta.device or not t.is_cuda):
                raise ValueError(f"{name}: expected contiguous {torch.float32} {(n,)} on one CUDA device, "
                                 f"got {t.dtype} {tuple(t.shape)} on {t.device}")
        self.d, self.n_axes, self.device = d, len(pairs), theta.device
        self._tensors = (theta, q_weight, k_weight)
        ptr = [0 if t is None else t.data_ptr() for t in self._tensors]
        self._c = dkv_norm_rope_t(*ptr, eps, int(bool(norm)), layout, len(pairs), (ctypes.c_int32 * 4)(*pairs))
        self._ref = ctypes.byref(self._c)


def norm_rope(Q: Optional[torch.Tensor], K: Optional[torch.Tensor], how: NormRope, coord: torch.Tensor,
              out: Optional[Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]] = None, stream=None):
    """Queries Q [H_q][rows][d] and keys K [H_k][rows][d] (either may be None) normed and rotated to the coordinates
    coord [n_axes][rows] (int32) of their rows: (Q', K'), new tensors or those of `out` (which may be the inputs)."""
    some = Q if Q is not None else K
    if some is None:
        raise ValueError("norm_rope: neither queries nor keys")
    rows, device, d = some.shape[1], some.device, how.d
    if how.device != device:
        raise ValueError(f"how: expected tensors on {device}, got {how.device}")
    _check_i32(coord, (how.n_axes, rows), "coord", device)
    raw, ctx = _on_stream(stream, device)
    Qo, Ko = out if out is not None else (None, None)
    q = k = (0, None, 0, 0, None, 0, 0)
    if Q is not None:
        heads = Q.shape[0]
        a = _check_rows(Q, heads, rows, d, device, "Q")
        if Qo is None:
            Qo, z = _empty(ctx, (heads, rows, d), torch.bfloat16, device), (rows * d, d)
        else:
            z = _check_rows(Qo, heads, rows, d, device, "out")
        q = (heads, Q.data_ptr(), a[0], a[1], Qo.data_ptr(), z[0], z[1])
    if K is not None:
        heads = K.shape[0]
        a = _check_rows(K, heads, rows, d, device, "K")
        if Ko is None:
            Ko, z = _empty(ctx, (heads, rows, d), torch.bfloat16, device), (rows * d, d)
        else:
            z = _check_rows(Ko, heads, rows, d, device, "out")
        k = (heads, K.data_ptr(), a[0], a[1], Ko.data_ptr(), z[0], z[1])
    call = lib().dkv_norm_rope
    if torch.cuda.current_device() == device.index:
        st = call(d, how._ref, coord.data_ptr(), rows, *q, *k, raw)
    else:
        with torch.cuda.device(device):
            st = call(d, how._ref, coord.data_ptr(), rows, *q, *k, raw)
    if st != DKV_OK:
        _check(st, "dkv_norm_rope")
    return (Qo if Q is not None else None), (Ko if K is not None else None)


def _on_stream(stream, device):
    """The stream of a call on a device, and a context in which torch allocates for it (None: the current one)."""
    if stream is None:
        return _raw_stream(device.index), None
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    return stream.cuda_stream, torch.cuda.stream(stream)


def _empty(ctx, shape, dtype, device):
    if ctx is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with ctx:
        return torch.empty(shape, dtype=dtype, device=device)


class Summaries:
    """8-bit mean keys of a cache's pages: code [n_pages][H][d] int8 and scale [n_pages][H] uint8, allocated or taken."""

    def __init__(self, cache: "PagedCache", code: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None):
        shape = (cache.n_pages, cache.H, cache.d)
        self.code = torch.zeros(shape, dtype=torch.int8, device=cache.device) if code is None else code
        self.scale = torch.full(shape[:2], 77, dtype=torch.uint8, device=cache.device) if scale is None else scale
        for t, want, dtype, name in ((self.code, shape, torch.int8, "code"), (self.scale, shape[:2], torch.uint8, "scale")):
            if t.dtype != dtype or tuple(t.shape) != want or not t.is_contiguous() or t.device != cache.device:
                raise ValueError(f"{name}: expected contiguous {dtype} {want} on {cache.device}, "
                                 f"got {t.dtype} {tuple(t.shape)} on {t.device}")
        self.shape, self.device = shape, cache.device
        self._c = dkv_cache_summaries_t(self.code.data_ptr(), self.scale.data_ptr())
        self._ref = ctypes.byref(self._c)


class PagedCache:
    """Keys and values of H heads in pages of page_len positions, bf16 or quantised to e4m3
    ("bf16" / "e4m3"): allocates the pages with torch, or takes them (k, v and, for e4m3, k_scale,
    v_scale), and drives the C ABI.  Packed tensors are [heads][rows][d] bf16 with any strides that
    are multiples of 8 between heads and rows; rows behind the last sequence's are not written, so in an
    output that a method allocates itself they hold nothing in particular.  All methods enqueue on the current (or given)
    stream; a call on another stream than the one its tensors were made on is ordered by the caller."""

    def __init__(self, H: int, d: int, page_len: int, n_pages: int, fmt: str = "bf16", device="cuda",
                 k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        if fmt not in _CACHE_FORMAT:
            raise ValueError(f"fmt: expected one of {sorted(_CACHE_FORMAT)}, got {fmt!r}")
        dev = k.device if k is not None else torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self.H, self.d, self.page_len, self.n_pages, self.fmt, self.device = H, d, page_len, n_pages, fmt, dev
        e4m3 = fmt == "e4m3"

        def pages(t, dtype, shape, name):
            if t is None:
                return torch.zeros(shape, dtype=torch.uint8 if dtype.itemsize == 1 else dtype, device=dev).view(dtype)
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != dev:
                raise ValueError(f"{name}: expected contiguous {dtype} {shape} on {dev}, "
                                 f"got {t.dtype} {tuple(t.shape)} on {t.device}")
            return t
        shape = (n_pages, H, page_len, d)
        self.k = pages(k, torch.float8_e4m3fn if e4m3 else torch.bfloat16, shape, "k")
        self.v = pages(v, torch.float8_e4m3fn if e4m3 else torch.bfloat16, shape, "v")
        self.k_scale = pages(k_scale, torch.uint8, shape[:3], "k_scale") if e4m3 else None
        self.v_scale = pages(v_scale, torch.uint8, shape[:3], "v_scale") if e4m3 else None
        self._status = torch.zeros(2, dtype=torch.int32, device=dev)
        bufs = dkv_cache_buffers_t(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr() if e4m3 else None,
                                   self.v_scale.data_ptr() if e4m3 else None, self._status.data_ptr())
        h = ctypes.c_void_p()
        with torch.cuda.device(dev):
            _check(lib().dkv_cache_create(ctypes.byref(h), H, d, page_len, n_pages, _CACHE_FORMAT[fmt],
                                          ctypes.byref(bufs)), "dkv_cache_create")
        self.handle = h.value
        self._plans: Dict[tuple, tuple] = {}
        L = lib()
        self._write, self._read, self._attend = L.dkv_cache_write, L.dkv_cache_read, L.dkv_cache_attend
        self._write_norm_rope, self._summarise = L.dkv_cache_write_norm_rope, L.dkv_cache_summarise
        self._fork, self._extend, self._release = L.dkv_cache_fork, L.dkv_cache_extend, L.dkv_cache_release
        self._compact, self._choose, self._attend_chosen = L.dkv_cache_compact, L.dkv_cache_choose, L.dkv_cache_attend_chosen

    def close(self):
        if getattr(self, "handle", None):
            lib().dkv_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _packed(self, t: torch.Tensor, heads: int, rows: int, name: str):
        return _check_rows(t, heads, rows, self.d, self.device, name)

    def _on(self, stream):
        return _on_stream(stream, self.device)

    def _new(self, ctx, shape, dtype):
        return _empty(ctx, shape, dtype, self.device)

    def _seqs(self, seqs: CacheSeqs):
        if seqs.device != self.device:
            raise ValueError(f"seqs: expected tensors on {self.device}, got {seqs.device}")
        return seqs._ref

    def write(self, K: torch.Tensor, V: torch.Tensor, seqs: CacheSeqs, stream=None) -> None:
        """The sequences' newest tokens K, V [H][rows][d] into their pages (quantised if fmt is e4m3)."""
        rows = K.shape[1]
        k, v = self._packed(K, self.H, rows, "K"), self._packed(V, self.H, rows, "V")
        s, _ = self._on(stream)
        st = self._write(self.handle, self._seqs(seqs), K.data_ptr(), V.data_ptr(), rows, k[0], k[1], v[0], v[1], s)
        if st != DKV_OK:
            _check(st, "dkv_cache_write")

    def read(self, seqs: CacheSeqs, first: torch.Tensor, rows: int, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
             stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Positions first[b], first[b] + 1, .. of every sequence as rows row_start[b] .. of K, V
        [H][rows][d]; positions that a sequence does not hold are zeros."""
        if first.dtype != torch.int32 or first.shape != (seqs.n_seq,) or not first.is_contiguous() or first.device != self.device:
            raise ValueError(f"first: expected contiguous {torch.int32} {(seqs.n_seq,)} on {self.device}")
        s, ctx = self._on(stream)
        if out is None:
            shape = (self.H, rows, self.d)
            K, V = self._new(ctx, shape, torch.bfloat16), self._new(ctx, shape, torch.bfloat16)
            k = v = (rows * self.d, self.d)
        else:
            K, V = out
            k, v = self._packed(K, self.H, rows, "K"), self._packed(V, self.H, rows, "V")
        st = self._read(self.handle, self._seqs(seqs), first.data_ptr(), K.data_ptr(), V.data_ptr(), rows, k[0], k[1], v[0],
                        v[1], s)
        if st != DKV_OK:
            _check(st, "dkv_cache_read")
        return K, V

    def attend(self, Q: torch.Tensor, seqs: CacheSeqs, window: int = 0, sinks: int = 0, block: int = 1,
               scale: Optional[float] = None, max_rows: Optional[int] = None, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
        """Attention of the sequences' newest tokens Q [H_q][rows][d] over their cached keys (the
        mask of dkv_cache_attend_t).  max_rows: the most tokens of any one sequence, 1 when every
        sequence brings one (default: all rows)."""
        Hq, rows = Q.shape[0], Q.shape[1]
        key = (seqs.n_seq, Hq, rows, scale, window, sinks, block, max_rows)
        plan = self._plans.get(key)
        if plan is None:
            plan = self._plan(key)
        size, most, how, _ = plan
        q = self._packed(Q, Hq, rows, "Q")
        s, ctx = self._on(stream)
        if out is None:
            out = self._new(ctx, (Hq, rows, self.d), torch.bfloat16)
        o = self._packed(out, Hq, rows, "out")
        scratch = self._new(ctx, size, torch.uint8)
        st = self._attend(self.handle, self._seqs(seqs), Q.data_ptr(), Hq, rows, q[0], q[1], out.data_ptr(), o[0], o[1],
                          how, scratch.data_ptr(), size, s)
        if st != DKV_OK:
            _check(st, "dkv_cache_attend")
        return out

    def _plan(self, key):
        """Scratch bytes and the C structure of an attend call's sizes and options, kept for the next one."""
        n_seq, Hq, rows, scale, window, sinks, block, max_rows = key
        if scale is not None and not scale > 0.0:
            raise ValueError("scale: expected a positive number")
        _check_32(window=window, sinks=sinks, block=block)
        most = rows if max_rows is None else min(int(max_rows), rows)
        size = int(lib().dkv_cache_attend_scratch_size(self.handle, n_seq, Hq, rows, most))
        how = dkv_cache_attend_t(0.0 if scale is None else scale, window, sinks, block, most)
        return self._keep_plan(key, (size, most, ctypes.byref(how), how))

    def _keep_plan(self, key, plan):
        if len(self._plans) > 4096:
            self._plans.clear()
        self._plans[key] = plan
        return plan

    def sync(self) -> None:
        _check(lib().dkv_cache_sync(self.handle), "dkv_cache_sync")

    # ------------------------------------------------------------- norm and rotation on the way in
    def write_norm_rope(self, Q: Optional[torch.Tensor], K: torch.Tensor, V: torch.Tensor, seqs: CacheSeqs, how: NormRope,
                        coord: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        stream=None) -> Optional[torch.Tensor]:
        """The sequences' newest tokens: keys K normed, rotated and written into their pages beside the values V, queries Q
        [H_q][rows][d] (or None) normed and rotated into `out` or a new tensor, which is returned.  coord [n_axes][rows]
        int32: the tokens' coordinates (None: their positions)."""
        rows = K.shape[1]
        if how.d != self.d or how.device != self.device:
            raise ValueError(f"how: expected one of d = {self.d} on {self.device}, got {how.d} on {how.device}")
        if coord is not None:
            _check_i32(coord, (how.n_axes, rows), "coord", self.device)
        k, v = self._packed(K, self.H, rows, "K"), self._packed(V, self.H, rows, "V")
        s, ctx = self._on(stream)
        queries = (0, None, 0, 0, None, 0, 0)
        if Q is not None:
            heads = Q.shape[0]
            q = self._packed(Q, heads, rows, "Q")
            if out is None:
                out, o = self._new(ctx, (heads, rows, self.d), torch.bfloat16), (rows * self.d, self.d)
            else:
                o = self._packed(out, heads, rows, "out")
            queries = (heads, Q.data_ptr(), q[0], q[1], out.data_ptr(), o[0], o[1])
        st = self._write_norm_rope(self.handle, self._seqs(seqs), how._ref, None if coord is None else coord.data_ptr(), rows,
                                   *queries, K.data_ptr(), k[0], k[1], V.data_ptr(), v[0], v[1], s)
        if st != DKV_OK:
            _check(st, "dkv_cache_write_norm_rope")
        return out if Q is not None else None

    # ------------------------------------------------------------- pages
    def new_refs(self) -> torch.Tensor:
        """Counts for the calls below: every page free."""
        return torch.zeros(self.n_pages, dtype=torch.int32, device=self.device)

    def _table(self, t: PageTable):
        if t.device != self.device:
            raise ValueError(f"table: expected tensors on {self.device}, got {t.device}")
        return t._ref

    def _refs(self, refs: torch.Tensor) -> int:
        _check_i32(refs, (self.n_pages,), "refs", self.device)
        return refs.data_ptr()

    def _scratch(self, call: str, n_seq: int) -> int:
        size = self._plans.get((call, n_seq))
        if size is None:
            size = self._keep_plan((call, n_seq), int(getattr(lib(), f"dkv_cache_{call}_scratch_size")(self.handle, n_seq)))
        return size

    def fork(self, refs: torch.Tensor, src: PageTable, parent: torch.Tensor, dst: PageTable, stream=None) -> None:
        """Sequence i of dst goes on from sequence parent[i] (int32, -1: empty) of src, sharing its pages; src is given up."""
        _check_i32(parent, (dst.n_seq,), "parent", self.device)
        s, _ = self._on(stream)
        st = self._fork(self.handle, self._refs(refs), self._table(src), parent.data_ptr(), self._table(dst), s)
        if st != DKV_OK:
            _check(st, "dkv_cache_fork")

    def extend(self, refs: torch.Tensor, seqs: PageTable, add: torch.Tensor, stream=None) -> None:
        """Room for add[b] (int32) more positions of every sequence: pages, lengths, and a copy of a shared last page."""
        _check_i32(add, (seqs.n_seq,), "add", self.device)
        s, ctx = self._on(stream)
        size = self._scratch("extend", seqs.n_seq)
        scratch = self._new(ctx, size, torch.uint8)
        st = self._extend(self.handle, self._refs(refs), self._table(seqs), add.data_ptr(), scratch.data_ptr(), size, s)
        if st != DKV_OK:
            _check(st, "dkv_cache_extend")

    def release(self, refs: torch.Tensor, seqs: PageTable, first: torch.Tensor, last: torch.Tensor, stream=None) -> None:
        """Gives back the pages whose positions all lie in [first[b], last[b]) (int32); last[b] >= seq_len[b] ends the sequence
        at first[b] (inside a page: its summary is made again by summarise from the new length - 1 on)."""
        _check_i32(first, (seqs.n_seq,), "first", self.device)
        _check_i32(last, (seqs.n_seq,), "last", self.device)
        s, _ = self._on(stream)
        st = self._release(self.handle, self._refs(refs), self._table(seqs), first.data_ptr(), last.data_ptr(), s)
        if st != DKV_OK:
            _check(st, "dkv_cache_release")

    def compact(self, refs: torch.Tensor, src: PageTable, keep: torch.Tensor, keep_start: torch.Tensor, dst: PageTable,
                stream=None) -> None:
        """Position i of sequence b of dst := position keep[keep_start[b] + i] of sequence b of src (int32); src is given up.
        Summaries of moved pages are made again by summarise(first=0)."""
        _check_i32(keep, (keep.numel(),), "keep", self.device)
        _check_i32(keep_start, (src.n_seq + 1,), "keep_start", self.device)
        s, ctx = self._on(stream)
        size = self._scratch("compact", src.n_seq)
        scratch = self._new(ctx, size, torch.uint8)
        st = self._compact(self.handle, self._refs(refs), self._table(src), keep.data_ptr(), keep.numel(), keep_start.data_ptr(),
                           self._table(dst), scratch.data_ptr(), size, s)
        if st != DKV_OK:
            _check(st, "dkv_cache_compact")

    # ------------------------------------------------------------- chosen pages
    def _sums(self, summaries: Summaries):
        if summaries.shape != (self.n_pages, self.H, self.d) or summaries.device != self.device:
            raise ValueError(f"summaries: expected those of a cache of {(self.n_pages, self.H, self.d)} on {self.device}, "
                             f"got {summaries.shape} on {summaries.device}")
        return summaries._ref

    def summarise(self, seqs: CacheSeqs, summaries: Summaries, first: Optional[torch.Tensor] = None, stream=None) -> None:
        """8-bit mean keys of the pages that hold positions from first[b] (int32; None: the newest tokens') on."""
        if first is not None:
            _check_i32(first, (seqs.n_seq,), "first", self.device)
        s, _ = self._on(stream)
        st = self._summarise(self.handle, self._seqs(seqs), None if first is None else first.data_ptr(), self._sums(summaries), s)
        if st != DKV_OK:
            _check(st, "dkv_cache_summarise")

    def choose(self, Q: torch.Tensor, seqs: CacheSeqs, summaries: Summaries, top: int, tile: int = 1, block: int = 1,
               sink_pages: int = 1, local_pages: int = 2, width: Optional[int] = None, out: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
        """Lists [H][rows // tile + n_seq][width] (int32, -1 behind the last page) of the pages that each tile of `tile` tokens
        attends to in each key head: sinks, local ones and the `top` best by their summaries (see dkv_cache_choose)."""
        Hq, rows = Q.shape[0], Q.shape[1]
        if width is None:
            width = max(1, sink_pages + local_pages + (tile + self.page_len - 2) // self.page_len + top)
        key = ("choose", tile, block, sink_pages, local_pages, top, width)
        plan = self._plans.get(key)
        if plan is None:
            _check_32(tile=tile, block=block, sink_pages=sink_pages, local_pages=local_pages, top=top, width=width)
            if tile < 1:
                raise ValueError(f"tile: expected a positive number, got {tile}")
            how = dkv_cache_choose_t(tile, block, sink_pages, local_pages, top, width)
            plan = self._keep_plan(key, (ctypes.byref(how), how))
        q = self._packed(Q, Hq, rows, "Q")
        s, ctx = self._on(stream)
        shape = (self.H, rows // tile + seqs.n_seq, width)
        if out is None:
            out = self._new(ctx, shape, torch.int32)
        else:
            _check_i32(out, shape, "out", self.device)
        st = self._choose(self.handle, self._seqs(seqs), self._sums(summaries), Q.data_ptr(), Hq, rows, q[0], q[1], plan[0],
                          out.data_ptr(), s)
        if st != DKV_OK:
            _check(st, "dkv_cache_choose")
        return out

    def attend_chosen(self, Q: torch.Tensor, seqs: CacheSeqs, lists: torch.Tensor, tile: int = 1, block: int = 1,
                      scale: Optional[float] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of the sequences' newest tokens Q [H_q][rows][d] over the pages that `lists` (as choose returns
        them, for the same tile) names for their tile and key head."""
        Hq, rows = Q.shape[0], Q.shape[1]
        width = lists.shape[-1]
        key = ("chosen", scale, tile, block, width)
        plan = self._plans.get(key)
        if plan is None:
            if scale is not None and not scale > 0.0:
                raise ValueError("scale: expected a positive number")
            _check_32(tile=tile, block=block)
            if tile < 1:
                raise ValueError(f"tile: expected a positive number, got {tile}")
            how = dkv_cache_chosen_t(0.0 if scale is None else scale, tile, block, width)
            plan = self._keep_plan(key, (ctypes.byref(how), how))
        _check_i32(lists, (self.H, rows // tile + seqs.n_seq, width), "lists", self.device)
        q = self._packed(Q, Hq, rows, "Q")
        s, ctx = self._on(stream)
        if out is None:
            out = self._new(ctx, (Hq, rows, self.d), torch.bfloat16)
        o = self._packed(out, Hq, rows, "out")
        st = self._attend_chosen(self.handle, self._seqs(seqs), Q.data_ptr(), Hq, rows, q[0], q[1], out.data_ptr(), o[0], o[1],
                                 lists.data_ptr(), plan[0], s)
        if st != DKV_OK:
            _check(st, "dkv_cache_attend_chosen")
        return out
