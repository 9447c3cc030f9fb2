"""Thin ctypes binding of the C ABI in include/mf.h.

Argument marshalling only: every step of the scoring path runs in the CUDA
library.  Device buffers are torch tensors (their ``data_ptr()``) and calls run
on torch's current CUDA stream.  Importing this module loads the compiled
library and raises if it is missing; there is no fallback.
"""
from __future__ import annotations

import array
import ctypes as C
import functools
import operator
import os
import struct

import numpy as np
import torch
from torch.autograd.graph import increment_version

from . import build as _build

LIB_PATH = _build.LIB_PATH

MF_OK, MF_EINVAL, MF_ENOMEM, MF_ECUDA, MF_EUNSUPPORTED, MF_ETIMEOUT, MF_EDEVICE = range(7)
MF_FP32, MF_BF16, MF_FP32_SIMT = 0, 1, 2
_PRECISIONS = {"fp32": MF_FP32, "bf16": MF_BF16, "fp32_simt": MF_FP32_SIMT}
EMPTY = (1 << 64) - 1

_EXPORTS = ["mf_status_string", "mf_last_error", "mf_create", "mf_destroy", "mf_space_size",
            "mf_set_objective", "mf_score_batch", "mf_search_range", "mf_search_exhaustive",
            "mf_ga_generation", "mf_ga_init", "mf_ga_step", "mf_ga_run", "mf_check_device_status",
            "mf_get_stats", "mf_search_exhaustive_noalloc", "mf_fc_set", "mf_fc_table", "mf_fc_search",
            "mf_vram_feasible", "mf_set_utility", "mf_fc_ga_run", "mf_debug_wait_test",
            "mf_recurrence_sizes", "mf_recurrence_forward", "mf_recurrence_backward",
            "mf_orthogonalize_workspace", "mf_orthogonalize", "mf_operators_status",
            "mf_debug_operators_wait_test", "mf_linear_attention_sizes", "mf_linear_attention_forward",
            "mf_linear_attention_backward", "mf_embedding_forward", "mf_embedding_workspace", "mf_embedding_backward",
            "mf_clip_workspace", "mf_clip_gradients"]


class MFError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        super().__init__(f"{where}: {_lib.mf_status_string(status).decode()} ({detail})")


class _Problem(C.Structure):
    _fields_ = [
        ("n_models", C.c_int32), ("n_options", C.c_void_p), ("d_local", C.c_int32),
        ("hidden1", C.c_int32), ("hidden2", C.c_int32),
        ("local_feats", C.c_void_p), ("demand", C.c_void_p), ("weights", C.c_void_p),
        ("agg_scale", C.c_void_p), ("sla", C.c_void_p), ("obj_w", C.c_void_p),
        ("vram_cap", C.c_float), ("soft_penalty", C.c_float),
        ("out_act", C.c_int32), ("objective", C.c_int32), ("precision", C.c_int32),
        ("device", C.c_int32),
    ]


class _Result(C.Structure):
    _fields_ = [("best_idx", C.c_uint64), ("best_score", C.c_float), ("feasible_count", C.c_uint64),
                ("k", C.c_int32), ("topk_idx", C.c_void_p), ("topk_score", C.c_void_p)]


class _Stats(C.Structure):
    _fields_ = [("h2d_bytes_create", C.c_uint64), ("d2h_bytes_last", C.c_uint64),
                ("kernel_launches_last", C.c_int32), ("score_launches_last", C.c_int32),
                ("score_ms_last", C.c_float), ("total_ms_last", C.c_float), ("scoring_path", C.c_int32)]


class _GAParams(C.Structure):
    _fields_ = [("pop", C.c_int32), ("gens", C.c_int32), ("tournament", C.c_int32),
                ("mutation_p", C.c_double), ("elitism", C.c_int32)]


class _FcParams(C.Structure):
    _fields_ = [("obs", C.c_void_p), ("variant", C.c_void_p), ("quality", C.c_void_p),
                ("f_min", C.c_void_p), ("f_max", C.c_void_p), ("omega", C.c_void_p), ("tau", C.c_void_p),
                ("reload_cost", C.c_void_p), ("prev_variant", C.c_void_p),
                ("alpha", C.c_float), ("beta", C.c_float), ("delta", C.c_float)]


class _FcGAParams(C.Structure):
    _fields_ = [("pop", C.c_int32), ("gens", C.c_int32), ("tournament", C.c_int32),
                ("crossover_p", C.c_double), ("mutation_p", C.c_double), ("elitism", C.c_int32),
                ("repair", C.c_int32)]


class _Seq(C.Structure):
    _fields_ = [("d_ptr", C.c_void_p), ("stride_batch", C.c_int64), ("stride_time", C.c_int64)]


_RECUR_HEAD = [("type", C.c_int32), ("batch", C.c_int64), ("time", C.c_int64), ("dim", C.c_int64),
               ("x", _Seq), ("z", _Seq), ("d_marks", C.c_void_p), ("marks_stride_batch", C.c_int64),
               ("marks_stride_time", C.c_int64)]


class _Recurrence(C.Structure):
    _fields_ = _RECUR_HEAD + [("d_h0", C.c_void_p), ("h", _Seq), ("d_last", C.c_void_p), ("d_saved", C.c_void_p),
                              ("d_status", C.c_void_p)]


class _RecurrenceGrad(C.Structure):
    _fields_ = _RECUR_HEAD + [("d_saved", C.c_void_p), ("dh", _Seq), ("d_dlast", C.c_void_p), ("dx", _Seq),
                              ("dz", _Seq), ("d_dh0", C.c_void_p), ("d_status", C.c_void_p)]


class _Orthogonalize(C.Structure):
    _fields_ = [("type", C.c_int32), ("batch", C.c_int64), ("rows", C.c_int64), ("cols", C.c_int64),
                ("d_g", C.c_void_p), ("g_stride_batch", C.c_int64), ("g_stride_row", C.c_int64),
                ("d_out", C.c_void_p), ("out_stride_batch", C.c_int64), ("out_stride_row", C.c_int64),
                ("steps", C.c_int32), ("a", C.c_float), ("b", C.c_float), ("c", C.c_float), ("eps", C.c_float),
                ("d_status", C.c_void_p)]


class _Heads(C.Structure):
    _fields_ = [("d_ptr", C.c_void_p), ("stride_batch", C.c_int64), ("stride_time", C.c_int64), ("stride_head", C.c_int64)]


_ATTEND_HEAD = [("type", C.c_int32), ("batch", C.c_int64), ("time", C.c_int64), ("heads", C.c_int64), ("dim_k", C.c_int64),
                ("dim_v", C.c_int64), ("q", _Heads), ("k", _Heads), ("v", _Heads), ("d_log_decay", C.c_void_p)]
_ATTEND_MARKS = [("d_marks", C.c_void_p), ("marks_stride_batch", C.c_int64), ("marks_stride_time", C.c_int64),
                 ("scale", C.c_float)]


class _LinearAttention(C.Structure):
    _fields_ = _ATTEND_HEAD + [("d_state", C.c_void_p)] + _ATTEND_MARKS + [
        ("o", _Heads), ("d_last", C.c_void_p), ("d_saved", C.c_void_p), ("d_status", C.c_void_p)]


class _LinearAttentionGrad(C.Structure):
    _fields_ = _ATTEND_HEAD + [("d_saved", C.c_void_p)] + _ATTEND_MARKS + [
        ("dout", _Heads), ("d_dlast", C.c_void_p), ("dq", _Heads), ("dk", _Heads), ("dv", _Heads),
        ("d_dstate", C.c_void_p), ("d_status", C.c_void_p)]


class _Embedding(C.Structure):
    _fields_ = [("type", C.c_int32), ("id_bits", C.c_int32), ("rows", C.c_int64), ("dim", C.c_int64), ("tokens", C.c_int64),
                ("d_table", C.c_void_p), ("table_stride", C.c_int64), ("d_ids", C.c_void_p), ("d_out", C.c_void_p),
                ("out_stride", C.c_int64), ("scale", C.c_float), ("d_status", C.c_void_p)]


class _EmbeddingGrad(C.Structure):
    _fields_ = [("type", C.c_int32), ("id_bits", C.c_int32), ("rows", C.c_int64), ("dim", C.c_int64), ("tokens", C.c_int64),
                ("d_dout", C.c_void_p), ("dout_stride", C.c_int64), ("d_ids", C.c_void_p), ("d_dtable", C.c_void_p),
                ("dtable_stride", C.c_int64), ("scale", C.c_float), ("d_status", C.c_void_p)]


class _Clip(C.Structure):
    _fields_ = [("count", C.c_int64), ("d_in", C.c_void_p), ("d_out", C.c_void_p), ("sizes", C.c_void_p),
                ("types", C.c_void_p), ("max_norm", C.c_float), ("eps", C.c_float), ("d_norm", C.c_void_p)]


# The same structures packed field by field (native sizes and alignment): a third of the time that a ctypes structure takes,
# which counts where a call takes 20 us.
_PACK_RECURRENCE = struct.Struct("@iqqq PqqPqqPqq PPqqPPP").pack
_PACK_RECURRENCE_GRAD = struct.Struct("@iqqq PqqPqqPqq PPqqP PqqPqq PP").pack
_PACK_ATTEND = struct.Struct("@iqqqqq PqqqPqqqPqqq PP Pqqf Pqqq PPP").pack
_PACK_ATTEND_GRAD = struct.Struct("@iqqqqq PqqqPqqqPqqq PP Pqqf Pqqq P PqqqPqqqPqqq PP").pack
_PACK_EMBEDDING = struct.Struct("@iiqqq PqP PqfP").pack  # (and of its gradient)
_PACK_CLIP = struct.Struct("@qPPPP ffP").pack
_PACK_ORTHOGONALIZE = struct.Struct("@iqqq PqqPqq iffff P").pack


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with paper_2609_02109_gb300.build.build()")
    lib = C.CDLL(LIB_PATH)
    vp, u64, i32, st = C.c_void_p, C.c_uint64, C.c_int32, C.c_int
    lib.mf_status_string.argtypes = [st]; lib.mf_status_string.restype = C.c_char_p
    lib.mf_last_error.argtypes = []; lib.mf_last_error.restype = C.c_char_p
    lib.mf_create.argtypes = [C.POINTER(_Problem), C.POINTER(vp)]
    lib.mf_destroy.argtypes = [vp]
    lib.mf_space_size.argtypes = [vp, C.POINTER(u64)]
    lib.mf_set_objective.argtypes = [vp, vp, vp]
    lib.mf_score_batch.argtypes = [vp, vp, u64, vp, vp, vp, vp]
    lib.mf_search_range.argtypes = [vp, u64, u64, i32, u64, C.POINTER(_Result), vp]
    lib.mf_search_exhaustive.argtypes = [vp, i32, u64, C.POINTER(_Result), vp]
    lib.mf_ga_generation.argtypes = [vp, vp, i32, vp, vp]
    lib.mf_ga_init.argtypes = [vp, C.POINTER(_GAParams), u64, vp, vp]
    lib.mf_ga_step.argtypes = [vp, C.POINTER(_GAParams), u64, i32, vp, vp, vp, vp]
    lib.mf_ga_run.argtypes = [vp, C.POINTER(_GAParams), u64, vp, vp, vp]
    lib.mf_check_device_status.argtypes = [vp, vp]
    lib.mf_debug_wait_test.argtypes = [vp, C.c_uint32]
    lib.mf_get_stats.argtypes = [vp, C.POINTER(_Stats)]
    lib.mf_search_exhaustive_noalloc.argtypes = [C.POINTER(_Problem), i32, u64, C.POINTER(_Result), vp]
    lib.mf_fc_set.argtypes = [vp, C.POINTER(_FcParams), vp]
    lib.mf_fc_table.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.mf_fc_search.argtypes = [vp, u64, u64, i32, u64, C.POINTER(_Result), vp]
    lib.mf_vram_feasible.argtypes = [vp, u64, u64, vp, u64, C.POINTER(u64), vp]
    lib.mf_set_utility.argtypes = [vp, C.POINTER(_FcParams)]
    lib.mf_fc_ga_run.argtypes = [vp, C.POINTER(_FcGAParams), u64, vp, vp, vp]
    lib.mf_recurrence_sizes.argtypes = [i32, C.c_int64, C.c_int64, C.c_int64, C.POINTER(u64), C.POINTER(u64),
                                        C.POINTER(u64)]
    # (arguments as ctypes structures by reference, or packed: see _PACK_RECURRENCE)
    lib.mf_recurrence_forward.argtypes = [vp, vp, u64, vp]
    lib.mf_recurrence_backward.argtypes = [vp, vp, u64, vp]
    lib.mf_orthogonalize_workspace.argtypes = [vp, C.POINTER(u64)]
    lib.mf_orthogonalize.argtypes = [vp, vp, u64, vp]
    lib.mf_linear_attention_sizes.argtypes = [i32] + [C.c_int64] * 5 + [C.POINTER(u64)] * 3
    lib.mf_linear_attention_forward.argtypes = [vp, vp, u64, vp]
    lib.mf_linear_attention_backward.argtypes = [vp, vp, u64, vp]
    lib.mf_embedding_forward.argtypes = [vp, vp]
    lib.mf_embedding_workspace.argtypes = [vp, C.POINTER(u64)]
    lib.mf_embedding_backward.argtypes = [vp, vp, u64, vp]
    lib.mf_clip_workspace.argtypes = [vp, C.POINTER(u64)]
    lib.mf_clip_gradients.argtypes = [vp, vp, u64, vp]
    lib.mf_operators_status.argtypes = [C.POINTER(vp)]
    lib.mf_debug_operators_wait_test.argtypes = [C.c_uint32]
    for name in _EXPORTS[2:]:
        getattr(lib, name).restype = st
    return lib


_lib = _load()


def lib() -> C.CDLL:
    return _lib


def _check(status: int, where: str):
    if status != MF_OK:
        raise MFError(status, where, _lib.mf_last_error().decode())


# The stream's address without the Stream object that torch.cuda.current_stream builds for it; a
# torch without this function is asked for the object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# And the current device without torch.cuda.current_device's check that CUDA is initialised (a tensor is there already).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(device) -> int:
    """torch's current stream on a device (an ordinal, or a tensor's device), as an address."""
    i = device if isinstance(device, int) else device.index
    return torch.cuda.current_stream(i).cuda_stream if _raw_stream is None else _raw_stream(i)


def _ptr(a) -> int:
    """Address of a numpy array (``a.ctypes`` builds an object for it on every use)."""
    return a.__array_interface__["data"][0]


def _search_result(k: int):
    """Result arrays of a search and the struct that points to them."""
    ti = np.empty(k, dtype=np.uint64)
    ts = np.empty(k, dtype=np.float32)
    return _Result(0, 0.0, 0, k, _ptr(ti), _ptr(ts)), ti, ts


def _as(a, dtype) -> np.ndarray:
    """`a` as a contiguous array of the type (itself where it is one)."""
    if type(a) is np.ndarray and a.dtype == dtype and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(a, dtype=dtype)


def _ga(params: dict) -> _GAParams:
    return _GAParams(int(params["pop"]), int(params["gens"]), int(params["tournament"]),
                     float(params["mutation_p"]), int(params.get("elitism", 1)))


def _f32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.float32)


def _problem_struct(prob: dict, device: int, prec: str):
    """mf_problem for a workload dict; returns (struct, arrays kept alive)."""
    keep = {
        "n_options": np.ascontiguousarray(prob["n_options"], dtype=np.int32),
        "local_feats": _f32(prob["local_feats"]), "demand": _f32(prob["demand"]),
        "weights": _f32(prob["weights"]),
        "agg_scale": None if prob.get("agg_scale") is None else _f32(prob["agg_scale"]),
        "sla": _f32(prob["sla"]), "obj_w": _f32(prob["obj_w"]),
    }
    ptr = lambda a: None if a is None else a.ctypes.data  # noqa: E731
    k = keep
    p = _Problem(int(k["n_options"].size), ptr(k["n_options"]), int(prob["d_local"]),
                 int(prob["hidden1"]), int(prob["hidden2"]), ptr(k["local_feats"]), ptr(k["demand"]),
                 ptr(k["weights"]), ptr(k["agg_scale"]), ptr(k["sla"]), ptr(k["obj_w"]),
                 float(prob["vram_cap"]), float(prob.get("soft_penalty", 0.0)),
                 1 if prob.get("out_act", "identity") == "sigmoid" else 0,
                 1 if prob.get("objective", "weighted_thr") == "soft_lat" else 0,
                 _PRECISIONS[prec], int(device))
    return p, keep


def search_exhaustive_noalloc(prob: dict, k: int, chunk: int = 0, device: int | None = None) -> dict:
    """mf_search_exhaustive_noalloc: the exact fp32 search with no device allocation
    (all device memory in the library's fixed array); same result fields as
    Context.search."""
    torch.cuda.init()  # (a no-op once done; the stream is asked for without it)
    device = torch.cuda.current_device() if device is None else int(device)
    p, _keep = _problem_struct(prob, device, "fp32")
    r, ti, ts = _search_result(k)
    _check(_lib.mf_search_exhaustive_noalloc(C.byref(p), int(k), int(chunk), C.byref(r),
                                              _stream(device)), "mf_search_exhaustive_noalloc")
    return dict(best_idx=int(r.best_idx), best_score=float(r.best_score),
                count=int(r.feasible_count), topk_idx=ti, topk_score=ts)


class Context:
    """An mf_ctx bound to one problem (a dict as drawn by ``workload``)."""

    def __init__(self, prob: dict, device: int | None = None, precision: str | None = None):
        self.device = torch.cuda.current_device() if device is None else int(device)
        prec = precision or prob.get("precision", "fp32")
        p, self._keep = _problem_struct(prob, self.device, prec)
        self.n_models = int(p.n_models)
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(_lib.mf_create(C.byref(p), C.byref(h)), "mf_create")
        self._h = h
        self.precision = prec
        v = C.c_uint64()  # (fixed for the context's life)
        _check(_lib.mf_space_size(self._h, C.byref(v)), "mf_space_size")
        self._space = int(v.value)

    # -- lifetime -----------------------------------------------------------------
    def close(self):
        if getattr(self, "_h", None):
            _lib.mf_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- calls ----------------------------------------------------------------------
    @property
    def space_size(self) -> int:
        if not self._h:  # (closed)
            raise MFError(MF_EINVAL, "mf_space_size", "NULL argument")
        return self._space

    def set_objective(self, sla=None, obj_w=None):
        s = None if sla is None else _f32(sla)
        w = None if obj_w is None else _f32(obj_w)
        _check(_lib.mf_set_objective(self._h, None if s is None else s.ctypes.data,
                                     None if w is None else w.ctypes.data), "mf_set_objective")

    def score_batch(self, idx: torch.Tensor, with_pred: bool = False, score=None, feasible=None,
                    pred=None):
        """idx: int64/uint64 CUDA tensor of joint indices -> (score f32, feasible u8[, pred])."""
        assert idx.is_cuda and idx.dtype in (torch.int64, torch.uint64) and idx.is_contiguous()
        n = idx.numel()
        dev = idx.device
        score = torch.empty(n, dtype=torch.float32, device=dev) if score is None else score
        feasible = torch.empty(n, dtype=torch.uint8, device=dev) if feasible is None else feasible
        if with_pred and pred is None:
            pred = torch.empty((n, self.n_models, 2), dtype=torch.float32, device=dev)
        _check(_lib.mf_score_batch(self._h, idx.data_ptr(), n, score.data_ptr(), feasible.data_ptr(),
                                   pred.data_ptr() if pred is not None else None, _stream(dev)),
               "mf_score_batch")
        return (score, feasible, pred) if with_pred else (score, feasible)

    def search(self, k: int, lo: int = 0, hi: int | None = None, chunk: int = 0) -> dict:
        hi = self.space_size if hi is None else int(hi)
        r, ti, ts = _search_result(k)
        _check(_lib.mf_search_range(self._h, int(lo), hi, int(k), int(chunk), C.byref(r),
                                    _stream(self.device)), "mf_search_range")
        return dict(best_idx=int(r.best_idx), best_score=float(r.best_score),
                    count=int(r.feasible_count), topk_idx=ti, topk_score=ts)

    def ga_generation(self, pop: torch.Tensor, fitness: torch.Tensor | None = None) -> torch.Tensor:
        assert pop.is_cuda and pop.dtype == torch.int32 and pop.is_contiguous()
        P = pop.shape[0]
        fitness = torch.empty(P, dtype=torch.float32, device=pop.device) if fitness is None else fitness
        _check(_lib.mf_ga_generation(self._h, pop.data_ptr(), P, fitness.data_ptr(), _stream(pop.device)),
               "mf_ga_generation")
        return fitness

    def ga_init(self, params: dict, seed: int) -> torch.Tensor:
        g = _ga(params)
        pop = torch.empty((g.pop, self.n_models), dtype=torch.int32, device=f"cuda:{self.device}")
        _check(_lib.mf_ga_init(self._h, C.byref(g), int(seed), pop.data_ptr(), _stream(pop.device)),
               "mf_ga_init")
        return pop

    def ga_step(self, params: dict, seed: int, gen: int, pop: torch.Tensor,
                fitness: torch.Tensor) -> torch.Tensor:
        g = _ga(params)
        nxt = torch.empty_like(pop)
        _check(_lib.mf_ga_step(self._h, C.byref(g), int(seed), int(gen), pop.data_ptr(),
                               fitness.data_ptr(), nxt.data_ptr(), _stream(pop.device)), "mf_ga_step")
        return nxt

    def ga_run(self, params: dict, seed: int):
        g = _ga(params)
        genome = np.zeros(self.n_models, dtype=np.int32)
        fit = C.c_float()
        _check(_lib.mf_ga_run(self._h, C.byref(g), int(seed), _ptr(genome), C.byref(fit),
                              _stream(self.device)), "mf_ga_run")
        return float(fit.value), genome

    # -- fixed-context mode ---------------------------------------------------
    @staticmethod
    def _fc_params(fc: dict):
        f, i = np.dtype(np.float32), np.dtype(np.int32)
        keep = [_as(fc[k], t) for k, t in (("obs", f), ("variant", i), ("quality", f), ("f_min", f), ("f_max", f),
                                           ("omega", f), ("tau", f), ("reload_cost", f), ("prev_variant", i))]
        p = _FcParams(*map(_ptr, keep), float(fc["alpha"]), float(fc["beta"]), float(fc["delta"]))
        return p, keep

    def fc_set(self, fc: dict) -> None:
        """Evaluate the local predictions under fc["obs"] and build the utility table."""
        p, keep = self._fc_params(fc)
        _check(_lib.mf_fc_set(self._h, C.byref(p), _stream(self.device)), "mf_fc_set")

    def set_utility(self, fc: dict | None) -> None:
        """Score with the Eq. 3 utility on the coupled aggregate (None: the problem's objective)."""
        if fc is None:
            _check(_lib.mf_set_utility(self._h, None), "mf_set_utility")
            return
        p, keep = self._fc_params(dict(fc, obs=np.zeros(4, np.float32)))
        _check(_lib.mf_set_utility(self._h, C.byref(p)), "mf_set_utility")

    def fc_table(self):
        """(fhat, f, u, ok) of every option row, as numpy arrays."""
        rows = int(self._keep["n_options"].sum())
        dev = f"cuda:{self.device}"
        fhat, f, u = (torch.empty(rows, dtype=torch.float32, device=dev) for _ in range(3))
        ok = torch.empty(rows, dtype=torch.uint8, device=dev)
        _check(_lib.mf_fc_table(self._h, fhat.data_ptr(), f.data_ptr(), u.data_ptr(), ok.data_ptr(),
                                _stream(self.device)), "mf_fc_table")
        torch.cuda.current_stream(self.device).synchronize()
        return fhat.cpu().numpy(), f.cpu().numpy(), u.cpu().numpy(), ok.cpu().numpy().astype(bool)

    def fc_search(self, k: int, lo: int = 0, hi: int | None = None, chunk: int = 0) -> dict:
        hi = self.space_size if hi is None else int(hi)
        r, ti, ts = _search_result(k)
        _check(_lib.mf_fc_search(self._h, int(lo), hi, int(k), int(chunk), C.byref(r), _stream(self.device)),
               "mf_fc_search")
        return dict(best_idx=int(r.best_idx), best_score=float(r.best_score), count=int(r.feasible_count),
                    topk_idx=ti, topk_score=ts)

    def fc_ga_run(self, params: dict, seed: int):
        """The paper's GA on the fixed-context landscape: (best J, genome)."""
        g = _FcGAParams(int(params["pop"]), int(params["gens"]), int(params["tournament"]),
                        float(params["crossover_p"]), float(params["mutation_p"]), int(params["elitism"]),
                        int(params["repair"]))
        genome = np.zeros(self.n_models, dtype=np.int32)
        fit = C.c_float()
        _check(_lib.mf_fc_ga_run(self._h, C.byref(g), int(seed), _ptr(genome), C.byref(fit),
                                 _stream(self.device)), "mf_fc_ga_run")
        return float(fit.value), genome

    def vram_feasible(self, lo: int = 0, hi: int | None = None, cap: int | None = None):
        """(count, device tensor of the first min(count, cap) VRAM-feasible indices)."""
        hi = self.space_size if hi is None else int(hi)
        cap = (hi - int(lo)) if cap is None else int(cap)
        out = torch.empty(max(cap, 1), dtype=torch.int64, device=f"cuda:{self.device}")
        cnt = C.c_uint64(0)
        _check(_lib.mf_vram_feasible(self._h, int(lo), hi, out.data_ptr(), cap, C.byref(cnt),
                                     _stream(self.device)), "mf_vram_feasible")
        c = int(cnt.value)
        return c, out[:min(c, cap)]

    def stats(self) -> dict:
        st = _Stats()
        _check(_lib.mf_get_stats(self._h, C.byref(st)), "mf_get_stats")
        return {f: getattr(st, f) for f, _ in _Stats._fields_}

    def check_status(self) -> int:
        """MF_OK, or the status of the first device-reported problem (clears it)."""
        return int(_lib.mf_check_device_status(self._h, _stream(self.device)))

    def debug_wait_test(self, polls: int) -> None:
        """mf_debug_wait_test: with polls > 0 the context's waiting kernels first wait on
        a flag that nothing sets and give up (tests of the timeout path); 0 restores."""
        _check(_lib.mf_debug_wait_test(self._h, int(polls)), "mf_debug_wait_test")


# -- operators that train the predictors and their monitor state -----------------
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # mf_type
MARK_MISSING, MARK_SAMPLE, MARK_FIRST = 0, 1, 2
NO_TOKEN = -1
_status_words: dict = {}  # device ordinal -> address of the word that bounded waits which give up set


def _refuse(where: str, detail: str):
    raise MFError(MF_EINVAL, where, detail)


def _status_word(device) -> int:
    """Address of the device's status word."""
    w = _status_words.get(device.index)
    if w is None:
        p = C.c_void_p()
        with torch.cuda.device(device):
            _check(_lib.mf_operators_status(C.byref(p)), "mf_operators_status")
        w = _status_words[device.index] = p.value
    return w


class _Word:
    """A device word by its address, for torch."""

    def __init__(self, address: int):
        self.__cuda_array_interface__ = {"shape": (1,), "typestr": "<i4", "data": (address, False), "version": 2}


def check_operators(device: int | None = None) -> int:
    """MF_OK, or MF_ETIMEOUT if a device-side wait of an operator gave up on the device since the last check, or
    MF_EDEVICE if embedding or embedding_backward saw an id that is neither a row of the table nor NO_TOKEN (waits
    for the device; clears the flag)."""
    torch.cuda.init()
    device = torch.cuda.current_device() if device is None else int(device)
    if device not in _status_words:
        return MF_OK
    w = torch.as_tensor(_Word(_status_words[device]), device=f"cuda:{device}")
    torch.cuda.synchronize(device)
    bad = int(w.item())
    w.zero_()
    return MF_ETIMEOUT if bad & ~1 else MF_EDEVICE if bad else MF_OK


def debug_operators_wait_test(polls: int) -> None:
    """mf_debug_operators_wait_test: with polls > 0 the waits of the calling thread's later operator calls expect
    what nothing sends and give up (tests of the timeout path); 0 restores."""
    _check(_lib.mf_debug_operators_wait_test(int(polls)), "mf_debug_operators_wait_test")


# (Tensors that a call writes in place get a new version, as torch's own in-place operations give them: a gradient that
# needs the old values raises then.)
def _call(where: str, fn, args: bytes, work_bytes: int, device) -> None:
    """fn(args, scratch, work_bytes, stream) on the device and its current stream; the scratch comes from torch's
    allocator, which keeps it for that stream."""
    if device.index != _current_device():
        with torch.cuda.device(device):
            return _call(where, fn, args, work_bytes, device)
    work = torch.empty(work_bytes, dtype=torch.uint8, device=device) if work_bytes else None
    _check(fn(args, work.data_ptr() if work_bytes else None, work_bytes, _stream(device)), where)


def _seq_of(where: str, name: str, t, like) -> tuple:
    """(address, batch stride, time stride) of a [batch, time, dim] tensor that goes with `like`."""
    if t is not like:
        if not isinstance(t, torch.Tensor) or t.shape != like.shape or t.dtype != like.dtype or t.device != like.device:
            _refuse(where, f"{name} must have the shape, type and device of x")
    sb, st, sd = t.stride()
    if sd != 1 and t.shape[2] > 1:
        _refuse(where, f"{name}: the last axis must be contiguous")
    return t.data_ptr(), sb, st


def _state_of(where: str, name: str, t, x, shape) -> int:
    """Address of a contiguous float32 tensor of the shape on x's device (None: 0)."""
    if t is None:
        return 0
    if (not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype != torch.float32 or t.device != x.device
            or not t.is_contiguous()):
        _refuse(where, f"{name} must be a contiguous float32 tensor of shape {tuple(shape)} on the device of x")
    return t.data_ptr()


def _recur_inputs(where: str, x, z, marks) -> tuple:
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dim() != 3 or x.dtype not in _TYPES:
        _refuse(where, "x must be a CUDA tensor [batch, time, dim] of float32, bfloat16 or float16")
    m = (0, 0, 0)
    if marks is not None:
        if (not isinstance(marks, torch.Tensor) or marks.shape != x.shape[:2] or marks.dtype != torch.uint8
                or marks.device != x.device):
            _refuse(where, "marks must be a uint8 tensor [batch, time] on the device of x")
        m = (marks.data_ptr(), *marks.stride())
    return (_TYPES[x.dtype], *x.shape, *_seq_of(where, "x", x, x), *_seq_of(where, "z", z, x), *m)


@functools.lru_cache(maxsize=256)
def _recur_sizes(device: int, kind: int, b: int, t: int, d: int) -> tuple:
    """(floats saved, scratch bytes forward, backward) of these sizes."""
    s, f, g = C.c_uint64(), C.c_uint64(), C.c_uint64()
    with torch.cuda.device(device):
        _check(_lib.mf_recurrence_sizes(kind, b, t, d, C.byref(s), C.byref(f), C.byref(g)), "mf_recurrence_sizes")
    return s.value, f.value, g.value


def recurrence(x: torch.Tensor, z: torch.Tensor, h0: torch.Tensor | None = None, marks: torch.Tensor | None = None,
               save: bool = False):
    """Gated linear recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t, f = sigmoid(z), along axis 1.

    x, z: [batch, time, dim] of one type (float32, bfloat16, float16), the last axis contiguous; h0:
    float32 [batch, dim] (None: zeros); marks: uint8 [batch, time] of MARK_MISSING, MARK_SAMPLE or
    MARK_FIRST (None: every step a sample).  Returns (h of x's type, the last state as float32), and
    with save=True also the tensor that recurrence_backward takes.  mf_recurrence_forward."""
    where = "mf_recurrence_forward"
    head = _recur_inputs(where, x, z, marks)
    kind, b, t, d = head[:4]
    dev = x.device
    h0p = _state_of(where, "h0", h0, x, (b, d))
    ns, nw, _ = _recur_sizes(dev.index, kind, b, t, d)
    h = torch.empty((b, t, d), dtype=x.dtype, device=dev)
    last = torch.empty((b, d), dtype=torch.float32, device=dev)
    saved = torch.empty(ns, dtype=torch.float32, device=dev) if save else None
    args = _PACK_RECURRENCE(*head, h0p, h.data_ptr(), t * d, d, last.data_ptr(), saved.data_ptr() if save else 0,
                            _status_word(dev))
    _call(where, _lib.mf_recurrence_forward, args, nw, dev)
    return (h, last, saved) if save else (h, last)


def recurrence_backward(dh: torch.Tensor, x: torch.Tensor, z: torch.Tensor, saved: torch.Tensor,
                        dlast: torch.Tensor | None = None, marks: torch.Tensor | None = None):
    """Gradients (dx, dz, dh0) of recurrence from those of h and (None: zeros) of the last state;
    x, z and marks as they were in the forward call, `saved` its third result.  mf_recurrence_backward."""
    where = "mf_recurrence_backward"
    head = _recur_inputs(where, x, z, marks)
    kind, b, t, d = head[:4]
    dev = x.device
    ns, _, nw = _recur_sizes(dev.index, kind, b, t, d)
    if saved is None:
        _refuse(where, "saved is required")
    savedp = _state_of(where, "saved", saved, x, (ns,))
    dlp = _state_of(where, "dlast", dlast, x, (b, d))
    g = _seq_of(where, "dh", dh, x)
    dx = torch.empty((b, t, d), dtype=x.dtype, device=dev)
    dz = torch.empty((b, t, d), dtype=x.dtype, device=dev)
    dh0 = torch.empty((b, d), dtype=torch.float32, device=dev)
    args = _PACK_RECURRENCE_GRAD(*head, savedp, *g, dlp, dx.data_ptr(), t * d, d, dz.data_ptr(), t * d, d, dh0.data_ptr(),
                                 _status_word(dev))
    _call(where, _lib.mf_recurrence_backward, args, nw, dev)
    return dx, dz, dh0


@functools.lru_cache(maxsize=256)
def _orth_bytes(device: int, kind: int, batch: int, rows: int, cols: int, steps: int, a: float, b: float, c: float,
                eps: float) -> int:
    """Scratch bytes of mf_orthogonalize for these sizes and coefficients, which it checks."""
    n = C.c_uint64()
    args = _PACK_ORTHOGONALIZE(kind, batch, rows, cols, 0, 0, 0, 0, 0, 0, steps, a, b, c, eps, 0)
    with torch.cuda.device(device):
        _check(_lib.mf_orthogonalize_workspace(args, C.byref(n)), "mf_orthogonalize")
    return n.value


def orthogonalize(g: torch.Tensor, steps: int = 5, coeffs=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """Newton-Schulz orthogonalisation of g[..., rows, cols] (float32, bfloat16 or float16): X = g / (|g|_F +
    eps), then `steps` times X <- a X + (b A + c A A) X with A = X X^T, on each matrix.  Rows or columns
    contiguous, the leading axes as one stride.  The result has g's type and shape (`out` if given, which
    may not overlap g).  mf_orthogonalize."""
    where = "mf_orthogonalize"
    if not isinstance(g, torch.Tensor) or not g.is_cuda or g.dim() < 2 or g.dtype not in _TYPES:
        _refuse(where, "g must be a CUDA tensor [..., rows, cols] of float32, bfloat16 or float16")
    dev = g.device
    if out is not None and (not isinstance(out, torch.Tensor) or out.shape != g.shape or out.dtype != g.dtype or out.device != dev):
        _refuse(where, "out must have the shape, type and device of g")
    # by columns where they are the contiguous axis: the transpose's result is the result's transpose
    flip = g.stride(-1) != 1 and g.stride(-2) == 1 and g.shape[-1] > 1
    if out is None:
        out = torch.empty(g.mT.shape if flip else g.shape, dtype=g.dtype, device=dev)
        out = out.mT if flip else out
    if not g.numel():
        return out
    gv, ov = (g.mT, out.mT) if flip else (g, out)
    if gv.dim() != 3:
        try:
            gv, ov = gv.view(-1, *gv.shape[-2:]), ov.view(-1, *ov.shape[-2:])
        except RuntimeError:
            _refuse(where, "the leading axes of g and out must view as one")
    batch, rows, cols = gv.shape
    gs, os_ = gv.stride(), ov.stride()
    if cols > 1 and (gs[2] != 1 or os_[2] != 1):
        _refuse(where, "g needs contiguous rows or columns, and out the same")
    a, b, c = map(float, coeffs)
    steps, eps, kind = int(steps), float(eps), _TYPES[g.dtype]
    n = _orth_bytes(dev.index, kind, batch, rows, cols, steps, a, b, c, eps)
    args = _PACK_ORTHOGONALIZE(kind, batch, rows, cols, gv.data_ptr(), gs[0], gs[1], ov.data_ptr(), os_[0], os_[1], steps,
                               a, b, c, eps, _status_word(dev))
    _call(where, _lib.mf_orthogonalize, args, n, dev)
    increment_version(out)
    return out


def _heads_of(where: str, name: str, t, like, dim: int) -> tuple:
    """(address, batch, time and head strides) of a [batch, time, heads, dim] tensor that goes with `like`."""
    if t is not like:
        if (not isinstance(t, torch.Tensor) or t.dim() != 4 or t.shape[:3] != like.shape[:3] or t.shape[3] != dim
                or t.dtype != like.dtype or t.device != like.device):
            _refuse(where, f"{name} must be [batch, time, heads, {dim}] of the type and on the device of q")
    sb, st, sh, sd = t.stride()
    if sd != 1 and dim > 1 and t.numel():
        _refuse(where, f"{name}: the last axis must be contiguous")
    return t.data_ptr(), sb, st, sh


def _attend_inputs(where: str, q, k, v, log_decay) -> tuple:
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 4 or q.dtype not in _TYPES:
        _refuse(where, "q must be a CUDA tensor [batch, time, heads, dim_k] of float32, bfloat16 or float16")
    if not isinstance(v, torch.Tensor) or v.dim() != 4:
        _refuse(where, "v must be a CUDA tensor [batch, time, heads, dim_v]")
    b, t, h, dk = q.shape
    dv = v.shape[3]
    return (_TYPES[q.dtype], b, t, h, dk, dv, *_heads_of(where, "q", q, q, dk), *_heads_of(where, "k", k, q, dk),
            *_heads_of(where, "v", v, q, dv), _required(where, "log_decay", log_decay, q, (h,)))


def _required(where: str, name: str, t, x, shape) -> int:
    if t is None:
        _refuse(where, f"{name} is required")
    return _state_of(where, name, t, x, shape)


def _marks_of(where: str, marks, q, shape) -> tuple:
    if marks is None:
        return 0, 0, 0
    if (not isinstance(marks, torch.Tensor) or marks.shape != shape or marks.dtype != torch.uint8
            or marks.device != q.device):
        _refuse(where, f"marks must be a uint8 tensor {list(shape)} on the device of q")
    return marks.data_ptr(), marks.stride(0), marks.stride(1) if marks.dim() > 1 else 0


@functools.lru_cache(maxsize=256)
def _attend_sizes(device: int, kind: int, b: int, t: int, h: int, dk: int, dv: int) -> tuple:
    """(floats saved, scratch bytes forward, backward) of these sizes."""
    s, f, g = C.c_uint64(), C.c_uint64(), C.c_uint64()
    with torch.cuda.device(device):
        _check(_lib.mf_linear_attention_sizes(kind, b, t, h, dk, dv, C.byref(s), C.byref(f), C.byref(g)),
               "mf_linear_attention_sizes")
    return s.value, f.value, g.value


def linear_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                     state: torch.Tensor | None = None, marks: torch.Tensor | None = None, scale: float = 1.0,
                     save: bool = False):
    """Linear attention S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t S_t, along axis 1.

    q, k: [batch, time, heads, dim_k], v: [batch, time, heads, dim_v] of one type (float32, bfloat16, float16), the last
    axis contiguous, dims at most 128; log_decay: float32 [heads]; state: float32 [batch, heads, dim_k, dim_v] (None:
    zeros); marks: uint8 [batch, time] of MARK_MISSING (the state stays, k and v are not used), MARK_SAMPLE or
    MARK_FIRST (the state before is dropped; None: every step a sample).  Returns (o of q's type, the last state as
    float32), and with save=True also the tensor that linear_attention_backward takes.  Sums are in float32; where bf16
    heads are wide, two of their operands have 16 bits (include/mf.h).  mf_linear_attention_forward."""
    where = "mf_linear_attention_forward"
    head = _attend_inputs(where, q, k, v, log_decay)
    kind, b, t, h, dk, dv = head[:6]
    dev = q.device
    statep = _state_of(where, "state", state, q, (b, h, dk, dv))
    m = _marks_of(where, marks, q, (b, t))
    ns, nw, _ = _attend_sizes(dev.index, kind, b, t, h, dk, dv)
    o = torch.empty((b, t, h, dv), dtype=q.dtype, device=dev)
    last = torch.empty((b, h, dk, dv), dtype=torch.float32, device=dev)
    saved = torch.empty(ns, dtype=torch.float32, device=dev) if save else None
    args = _PACK_ATTEND(*head, statep, *m, float(scale), o.data_ptr(), t * h * dv, h * dv, dv, last.data_ptr(),
                        saved.data_ptr() if save else 0, _status_word(dev))
    _call(where, _lib.mf_linear_attention_forward, args, nw, dev)
    return (o, last, saved) if save else (o, last)


def linear_attention_backward(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              log_decay: torch.Tensor, saved: torch.Tensor, dlast: torch.Tensor | None = None,
                              marks: torch.Tensor | None = None, scale: float = 1.0):
    """Gradients (dq, dk, dv, dstate) of linear_attention from those of o and (None: zeros) of the last state; the
    other arguments as they were in the forward call, `saved` its third result.  The decays are constants.
    mf_linear_attention_backward."""
    where = "mf_linear_attention_backward"
    head = _attend_inputs(where, q, k, v, log_decay)
    kind, b, t, h, dk, dv = head[:6]
    dev = q.device
    ns, _, nw = _attend_sizes(dev.index, kind, b, t, h, dk, dv)
    savedp = _required(where, "saved", saved, q, (ns,))
    dlp = _state_of(where, "dlast", dlast, q, (b, h, dk, dv))
    m = _marks_of(where, marks, q, (b, t))
    g = _heads_of(where, "do", do, q, dv)
    dq, dkey = (torch.empty((b, t, h, dk), dtype=q.dtype, device=dev) for _ in range(2))
    dvalue = torch.empty((b, t, h, dv), dtype=q.dtype, device=dev)
    dstate = torch.empty((b, h, dk, dv), dtype=torch.float32, device=dev)
    ks, vs = (t * h * dk, h * dk, dk), (t * h * dv, h * dv, dv)
    args = _PACK_ATTEND_GRAD(*head, savedp, *m, float(scale), *g, dlp, dq.data_ptr(), *ks, dkey.data_ptr(), *ks,
                             dvalue.data_ptr(), *vs, dstate.data_ptr(), _status_word(dev))
    _call(where, _lib.mf_linear_attention_backward, args, nw, dev)
    return dq, dkey, dvalue, dstate


def linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor,
                          state: torch.Tensor, marks: torch.Tensor | None = None, scale: float = 1.0) -> torch.Tensor:
    """One step of linear_attention for each row of a batch, as a server of many sequences takes it: q, k [batch,
    heads, dim_k], v [batch, heads, dim_v]; `state` (float32 [batch, heads, dim_k, dim_v]) is updated in place, not at
    all where marks (uint8 [batch]) say MARK_MISSING.  Returns o [batch, heads, dim_v]."""
    where = "mf_linear_attention_forward"
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3 \
            or not isinstance(v, torch.Tensor) or v.dim() != 3:
        _refuse(where, "q, k and v must be CUDA tensors [batch, heads, dim]")
    if not q.is_cuda or q.dtype not in _TYPES:
        _refuse(where, "q must be a CUDA tensor [batch, heads, dim_k] of float32, bfloat16 or float16")
    b, h, dk = q.shape
    dv, t, kind = v.shape[2], 1, _TYPES[q.dtype]
    seqs = []
    for name, x, d in (("q", q, dk), ("k", k, dk), ("v", v, dv)):
        if x.shape != (b, h, d) or x.dtype != q.dtype or x.device != q.device:
            _refuse(where, f"{name} must be [batch, heads, {d}] of the type and on the device of q")
        sb, sh, sd = x.stride()
        if sd != 1 and d > 1 and x.numel():
            _refuse(where, f"{name}: the last axis must be contiguous")
        seqs += x.data_ptr(), sb, 0, sh
    head = (kind, b, t, h, dk, dv, *seqs, _required(where, "log_decay", log_decay, q, (h,)))
    dev = q.device
    statep = _required(where, "state", state, q, (b, h, dk, dv))
    if state.requires_grad and torch.is_grad_enabled():
        _refuse(where, "state is updated in place, and must not require a gradient")
    m = _marks_of(where, marks, q, (b,))
    nw = _attend_sizes(dev.index, kind, b, t, h, dk, dv)[1]
    o = torch.empty((b, h, dv), dtype=q.dtype, device=dev)
    args = _PACK_ATTEND(*head, statep, *m, float(scale), o.data_ptr(), h * dv, h * dv, dv, statep, 0, _status_word(dev))
    _call(where, _lib.mf_linear_attention_forward, args, nw, dev)
    increment_version(state)
    return o


def _ids_of(where: str, ids, like) -> tuple:
    """(bits, number, address) of ids that go with a tensor."""
    if not isinstance(ids, torch.Tensor) or ids.dtype not in (torch.int32, torch.int64) or ids.device != like.device:
        _refuse(where, "ids must be an int32 or int64 tensor on the device of the other tensors")
    if not ids.is_contiguous():
        _refuse(where, "ids must be contiguous")
    return (64 if ids.dtype == torch.int64 else 32), ids.numel(), ids.data_ptr()


def embedding(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """out[..., :] = scale * table[ids[...]], zeros where an id is NO_TOKEN (-1).

    table: [rows, dim] (float32, bfloat16 or float16), rows contiguous; ids: int32 or int64, contiguous.  Any other id
    outside the table gives zeros too, and check_operators says so.  mf_embedding_forward."""
    where = "mf_embedding_forward"
    if not isinstance(table, torch.Tensor) or not table.is_cuda or table.dim() != 2 or table.dtype not in _TYPES:
        _refuse(where, "table must be a CUDA tensor [rows, dim] of float32, bfloat16 or float16")
    bits, n, idp = _ids_of(where, ids, table)
    rows, dim = table.shape
    if table.stride(1) != 1 and dim > 1 and table.numel():
        _refuse(where, "table: rows must be contiguous")
    dev = table.device
    out = torch.empty((*ids.shape, dim), dtype=table.dtype, device=dev)
    args = _PACK_EMBEDDING(_TYPES[table.dtype], bits, rows, dim, n, table.data_ptr(), table.stride(0), idp, out.data_ptr(),
                           dim, float(scale), _status_word(dev))
    _call(where, lambda a, work, size, stream: _lib.mf_embedding_forward(a, stream), args, 0, dev)
    return out


def embedding_backward(dout: torch.Tensor, ids: torch.Tensor, rows: int, scale: float = 1.0) -> torch.Tensor:
    """The gradient [rows, dim] of embedding's table from that of its result: scale times the sum of dout[..., :]
    over the places of each row, in fp32, rounded once to dout's type.  The same ids and scale as in the forward call;
    equal calls give equal bits.  mf_embedding_backward."""
    where = "mf_embedding_backward"
    if not isinstance(dout, torch.Tensor) or not dout.is_cuda or dout.dim() < 1 or dout.dtype not in _TYPES:
        _refuse(where, "dout must be a CUDA tensor [..., dim] of float32, bfloat16 or float16")
    bits, n, idp = _ids_of(where, ids, dout)
    if dout.shape[:-1] != ids.shape:
        _refuse(where, "dout must have the shape of ids, and an axis more")
    dim, rows = dout.shape[-1], int(rows)
    if dout.dim() != 2:
        try:
            dout = dout.view(n, dim)
        except RuntimeError:
            _refuse(where, "the leading axes of dout must view as one")
    if dout.stride(1) != 1 and dim > 1 and n:
        _refuse(where, "dout: the last axis must be contiguous")
    if rows < 0:
        _refuse(where, "rows must not be negative")
    dev = dout.device
    out = torch.empty((rows, dim), dtype=dout.dtype, device=dev)
    args = _PACK_EMBEDDING(_TYPES[dout.dtype], bits, rows, dim, n, dout.data_ptr(), dout.stride(0), idp, out.data_ptr(), dim,
                           float(scale), _status_word(dev))
    need = C.c_uint64()
    _check(_lib.mf_embedding_workspace(args, C.byref(need)), where)
    _call(where, _lib.mf_embedding_backward, args, need.value, dev)
    return out


def _dense(t: torch.Tensor) -> bool:
    """Whether a tensor's values fill its memory, in some order of its axes."""
    if t.is_contiguous():
        return True
    size = 1
    for stride, n in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride != size:
            return False
        size *= n
    return True


_DTYPE, _REQUIRES_GRAD = operator.attrgetter("dtype"), operator.attrgetter("requires_grad")


def _alike(a: torch.Tensor, b: torch.Tensor) -> bool:
    return a.shape == b.shape and a.stride() == b.stride()


def _tensors_of(where: str, tensors: list) -> tuple:
    """(types, addresses, sizes) of tensors that fill their memory, as arrays, and whether all are contiguous.  (By maps: a
    call may have thousands.)"""
    try:
        addresses = array.array("Q", map(torch.Tensor.data_ptr, tensors))
    except TypeError:
        _refuse(where, "grads and out must be tensors")
    try:
        kinds = array.array("i", map(_TYPES.__getitem__, map(_DTYPE, tensors)))
    except KeyError:
        _refuse(where, "grads must be float32, bfloat16 or float16")
    plain = all(map(torch.Tensor.is_contiguous, tensors))
    if not plain and not all(map(_dense, tensors)):
        _refuse(where, "a tensor does not fill its memory")
    return kinds, addresses, array.array("q", map(torch.Tensor.numel, tensors)), plain


def clip_gradients(grads, max_norm: float, eps: float = 1e-6, out=None) -> torch.Tensor:
    """Scales all tensors by min(1, max_norm / (norm + eps)), norm = sqrt(the sum of all values' squares), in place or
    into `out` (tensors of the same types and sizes, and of the same strides or contiguous as they are).  Returns the norm (a float32 scalar on the device, a sum of float32 sums).  A norm
    that is not finite scales nothing.

    grads: a sequence of CUDA tensors of one device (float32, bfloat16, float16, also mixed), each filling its memory
    in some order of its axes, none overlapping another.  max_norm = inf: the norm alone.  mf_clip_gradients."""
    where = "mf_clip_gradients"
    grads = list(grads)
    kinds, ins, sizes, plain = _tensors_of(where, grads)
    devices = set(map(torch.Tensor.get_device, grads))
    if len(devices) > 1 or -1 in devices:
        _refuse(where, "grads must be CUDA tensors of one device")
    dev = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
    if out is None:
        outs, written = ins, grads
    else:
        written = list(out)
        if len(written) != len(grads):
            _refuse(where, "out must have as many tensors")
        out_kinds, outs, out_sizes, out_plain = _tensors_of(where, written)
        if (out_kinds != kinds or out_sizes != sizes or set(map(torch.Tensor.get_device, written)) != devices
                or not (plain and out_plain or all(map(_alike, written, grads)))):
            _refuse(where, "out must have the tensors' sizes, types, strides and device")
    if torch.is_grad_enabled() and any(map(_REQUIRES_GRAD, written)):
        _refuse(where, "tensors that are written must not require a gradient")
    norm = torch.empty((), dtype=torch.float32, device=dev)
    args = _PACK_CLIP(len(grads), ins.buffer_info()[0], outs.buffer_info()[0], sizes.buffer_info()[0],
                      kinds.buffer_info()[0], float(max_norm), float(eps), norm.data_ptr())
    need = C.c_uint64()
    _check(_lib.mf_clip_workspace(args, C.byref(need)), where)
    _call(where, _lib.mf_clip_gradients, args, need.value, dev)
    increment_version(written)
    return norm
