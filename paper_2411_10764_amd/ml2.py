"""ctypes binding of the C ABI in include/ml2.h (argument marshalling only).

Every call goes straight to ``libml2.so``; all arithmetic runs in its HIP
kernels.  Device buffers are torch tensors (``tensor.data_ptr()``) or raw
integer device addresses; the stream defaults to torch's current stream.
The library must have been built (``python -m paper_2411_10764_amd.build``):
there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libml2.so")

ML2_OK = 0
ML2_ERR_INVALID_ARG = 1
ML2_ERR_UNSUPPORTED = 2
ML2_ERR_OUT_OF_MEMORY = 3
ML2_ERR_HIP = 4
ML2_MAX_DEPTH = 32
ML2_MAX_TREE_NODES = 3062
ML2_MAX_FEATURES = 256
ML2_MAX_TOPK = 16384
ML2_MAX_STREAM_K = 4096
ML2_MAX_ROWS = 2097152
ML2_MAX_TOKENS = 1073741824
ML2_MAX_WIDTH = 65536
ML2_MAX_TENSORS = 65536
ML2_STATE_BLOCK = 256
ML2_F32, ML2_BF16, ML2_F16 = 0, 1, 2

EXPORTED = (
    "ml2_load_ensemble", "ml2_free_ensemble", "ml2_ensemble_num_features",
    "ml2_ensemble_num_trees", "ml2_ensemble_depth", "ml2_score_validity",
    "ml2_score_perf", "ml2_score", "ml2_score_single_pass", "ml2_topk_workspace_bytes", "ml2_filter_topk", "ml2_filter_topk_noalloc",
    "ml2_rerank",
    "ml2_rerank_workspace_bytes",
    "ml2_explorer_create", "ml2_explorer_free", "ml2_explorer_reset", "ml2_explorer_rounds",
    "ml2_explorer_round", "ml2_stream_explorer_create", "ml2_stream_explorer_free",
    "ml2_stream_explorer_reset", "ml2_stream_explorer_rounds", "ml2_stream_explorer_begin",
    "ml2_stream_explorer_chunk", "ml2_stream_explorer_end", "ml2_last_error",
    "ml2_sample_workspace_bytes", "ml2_sample", "ml2_logprob_workspace_bytes", "ml2_logprob",
    "ml2_logprob_grad", "ml2_embed", "ml2_embed_grad_workspace_bytes", "ml2_embed_grad",
    "ml2_layer_norm", "ml2_layer_norm_grad_workspace_bytes", "ml2_layer_norm_grad",
    "ml2_grad_norm_workspace_bytes", "ml2_grad_norm", "ml2_adamw_state_bytes", "ml2_adamw",
)
# include/ml2_probe.h: microbenchmarks behind the roofline figures
EXPORTED_PROBE = ("ml2_probe_visit", "ml2_probe_lds", "ml2_probe_valu", "ml2_tune_walk_plan",
                  "ml2_tune_layout", "ml2_probe_walk")


class Ml2Error(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"ml2 status {status}: {message}")
        self.status = status


class ml2_ensemble_desc(ctypes.Structure):
    _fields_ = [
        ("num_trees", ctypes.c_int32),
        ("num_features", ctypes.c_int32),
        ("base_score", ctypes.c_float),
        ("tree_node_offset", ctypes.c_void_p),
        ("left_child", ctypes.c_void_p),
        ("right_child", ctypes.c_void_p),
        ("split_feature", ctypes.c_void_p),
        ("split_threshold", ctypes.c_void_p),
        ("leaf_value", ctypes.c_void_p),
        ("default_left", ctypes.c_void_p),
    ]


class ml2_adamw_tensor(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in
                ("param", "grad", "m", "v", "param_out", "m_out", "v_out", "copy")] + [
        ("n", ctypes.c_int64), ("weight_decay", ctypes.c_float)]


class ml2_adamw_options(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("lr_device", ctypes.c_void_p),
                ("step_device", ctypes.c_void_p), ("factor", ctypes.c_void_p),
                ("seed", ctypes.c_uint64)]


class ml2_walk_info(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in
                ("loaded", "codes", "mode", "depth", "waves", "per_cu", "group")]


_lib = None


def lib():
    """The loaded libml2.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2411_10764_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.ml2_load_ensemble.restype = I32
        L.ml2_load_ensemble.argtypes = [P, ctypes.POINTER(P)]
        L.ml2_free_ensemble.restype = None
        L.ml2_free_ensemble.argtypes = [P]
        for f in ("ml2_ensemble_num_features", "ml2_ensemble_num_trees", "ml2_ensemble_depth"):
            getattr(L, f).restype = I32
            getattr(L, f).argtypes = [P]
        L.ml2_score_validity.restype = I32
        L.ml2_score_validity.argtypes = [P, P, I64, I64, P, P, P]
        L.ml2_score_perf.restype = I32
        L.ml2_score_perf.argtypes = [P, P, I64, I64, P, P, P]
        L.ml2_score.restype = I32
        L.ml2_score.argtypes = [P, P, P, I64, I64, P, P, P, P]
        L.ml2_score_single_pass.restype = I32
        L.ml2_score_single_pass.argtypes = [P, P, P, I64, I64]
        L.ml2_topk_workspace_bytes.restype = I32
        L.ml2_topk_workspace_bytes.argtypes = [I64, I32, ctypes.POINTER(SZ)]
        L.ml2_filter_topk.restype = I32
        L.ml2_filter_topk.argtypes = [P, P, I64, I32, P, P, P, P, SZ, P]
        L.ml2_filter_topk_noalloc.restype = I32
        L.ml2_filter_topk_noalloc.argtypes = [P, P, I64, I32, P, P, P, P]
        L.ml2_rerank.restype = I32
        L.ml2_rerank.argtypes = [P, P, I64, I64, P, I32, I32, P, P, P, P, P, SZ, P]
        L.ml2_rerank_workspace_bytes.restype = I32
        L.ml2_rerank_workspace_bytes.argtypes = [P, I32, ctypes.POINTER(SZ)]
        L.ml2_explorer_create.restype = I32
        L.ml2_explorer_create.argtypes = [P, P, P, I64, I32, I32, I32, ctypes.POINTER(P)]
        L.ml2_explorer_free.restype = None
        L.ml2_explorer_free.argtypes = [P]
        L.ml2_explorer_reset.restype = I32
        L.ml2_explorer_reset.argtypes = [P]
        L.ml2_explorer_rounds.restype = I32
        L.ml2_explorer_rounds.argtypes = [P]
        L.ml2_explorer_round.restype = I32
        L.ml2_explorer_round.argtypes = [P, P, I64, I32, P, P, P, P]
        L.ml2_stream_explorer_create.restype = I32
        L.ml2_stream_explorer_create.argtypes = [P, P, P, I64, I32, I32, I32, ctypes.POINTER(P)]
        L.ml2_stream_explorer_free.restype = None
        L.ml2_stream_explorer_free.argtypes = [P]
        L.ml2_stream_explorer_reset.restype = I32
        L.ml2_stream_explorer_reset.argtypes = [P]
        L.ml2_stream_explorer_rounds.restype = I32
        L.ml2_stream_explorer_rounds.argtypes = [P]
        L.ml2_stream_explorer_begin.restype = I32
        L.ml2_stream_explorer_begin.argtypes = [P, P]
        L.ml2_stream_explorer_chunk.restype = I32
        L.ml2_stream_explorer_chunk.argtypes = [P, P, I64, I64, I64, P]
        L.ml2_stream_explorer_end.restype = I32
        L.ml2_stream_explorer_end.argtypes = [P, P, P, P, P]
        F32 = ctypes.c_float
        for f, types in (
                ("ml2_sample_workspace_bytes", [I64, I64, I32, ctypes.POINTER(SZ)]),
                ("ml2_sample", [I32, P, I64, I64, I64, P, I64, P, P, P, P, P, I32, P, P, P, SZ, P]),
                ("ml2_logprob_workspace_bytes", [I64, I64, I32, ctypes.POINTER(SZ)]),
                ("ml2_logprob", [I32, P, I64, I64, I64, P, I64, P, P, I32, P, P, SZ, P]),
                ("ml2_logprob_grad", [I32, P, I64, I64, I64, P, I64, P, P, P, I32, P, P, I64, P,
                                      SZ, P]),
                ("ml2_embed", [I32, P, I64, I64, I64, P, I64, F32, P, I64, P]),
                ("ml2_embed_grad_workspace_bytes", [I64, I64, I64, ctypes.POINTER(SZ)]),
                ("ml2_embed_grad", [I32, P, I64, I64, I64, P, F32, I32, P, I64, I64, P, SZ, P]),
                ("ml2_layer_norm", [I32, P, I64, I64, I64, I32, P, P, F32, P, I64, P, P, P]),
                ("ml2_layer_norm_grad_workspace_bytes", [I64, I64, ctypes.POINTER(SZ)]),
                ("ml2_layer_norm_grad", [I32, P, I64, I64, I64, P, I64, I32, P, P, P, P, I64, I32,
                                         P, P, P, SZ, P]),
                ("ml2_grad_norm_workspace_bytes", [P, I32, ctypes.POINTER(SZ)]),
                ("ml2_grad_norm", [I32, P, P, I32, F32, F32, P, P, P, P, SZ, P]),
                ("ml2_adamw_state_bytes", [I32, I64, ctypes.POINTER(SZ)]),
                ("ml2_adamw", [I32, I32, I32, P, I32, P, P])):
            getattr(L, f).restype = I32
            getattr(L, f).argtypes = types
        L.ml2_last_error.restype = ctypes.c_char_p
        L.ml2_last_error.argtypes = []
        D = ctypes.POINTER(ctypes.c_double)
        L.ml2_probe_visit.restype = I32
        L.ml2_probe_visit.argtypes = [I32, I32, I32, I32, I32, I32, I32, D, D]
        L.ml2_probe_lds.restype = I32
        L.ml2_probe_lds.argtypes = [I32, I32, I32, D, D]
        L.ml2_probe_valu.restype = I32
        L.ml2_probe_valu.argtypes = [I32, I32, D, D]
        L.ml2_tune_walk_plan.restype = I32
        L.ml2_tune_walk_plan.argtypes = [I32, I32, I32, I32, I32]
        L.ml2_tune_layout.restype = I32
        L.ml2_tune_layout.argtypes = [I32]
        L.ml2_probe_walk.restype = I32
        L.ml2_probe_walk.argtypes = [P, P, I64, I64, I32, I32, ctypes.POINTER(ml2_walk_info)]
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != ML2_OK:
        msg = lib().ml2_last_error()
        raise Ml2Error(status, msg.decode() if msg else "")


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        # torch.cuda.current_stream() makes an object first, which takes longer
        # than the rest of a call
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _rows(X):
    """(pointer, n, ld) of a 2-D row-major float32 device tensor."""
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be a 2-D tensor with unit column stride")
    return X.data_ptr(), X.shape[0], X.stride(0)


class Ensemble:
    """An ensemble loaded on the current device (owns the library handle)."""

    def __init__(self, handle: int):
        self.handle = handle

    @property
    def num_features(self) -> int:
        return lib().ml2_ensemble_num_features(self.handle)

    @property
    def num_trees(self) -> int:
        return lib().ml2_ensemble_num_trees(self.handle)

    @property
    def depth(self) -> int:
        return lib().ml2_ensemble_depth(self.handle)

    def free(self) -> None:
        if self.handle:
            lib().ml2_free_ensemble(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover - interpreter shutdown order
        try:
            self.free()
        except Exception:
            pass


def make_desc(ens):
    """(descriptor, keep-alive arrays) from a gen.Ensemble-like object."""
    arrays = (
        np.ascontiguousarray(ens.offsets, np.int64),
        np.ascontiguousarray(ens.left, np.int32),
        np.ascontiguousarray(ens.right, np.int32),
        np.ascontiguousarray(ens.feature, np.int32),
        np.ascontiguousarray(ens.threshold, np.float32),
        np.ascontiguousarray(ens.value, np.float32),
    )
    dl = getattr(ens, "default_left", None)
    if dl is not None:
        dl = np.ascontiguousarray(dl, np.uint8)
        arrays = arrays + (dl,)
    off, left, right, feat, thr, val = arrays[:6]
    d = ml2_ensemble_desc(int(off.shape[0] - 1), int(ens.num_features), float(ens.base_score),
                          off.ctypes.data, left.ctypes.data, right.ctypes.data,
                          feat.ctypes.data, thr.ctypes.data, val.ctypes.data,
                          None if dl is None else dl.ctypes.data)
    return d, arrays


def ml2_load_ensemble(ens) -> Ensemble:
    """Load a gen.Ensemble-like tree ensemble (or an ml2_ensemble_desc)."""
    if isinstance(ens, ml2_ensemble_desc):
        d, keep = ens, None
    else:
        d, keep = make_desc(ens)
    h = ctypes.c_void_p()
    _check(lib().ml2_load_ensemble(ctypes.byref(d), ctypes.byref(h)))
    del keep
    return Ensemble(h.value)


def ml2_free_ensemble(e: Ensemble) -> None:
    e.free()


def ml2_score_validity(v: Ensemble, X, valid_out, margin_out=None, stream=None) -> None:
    xp, n, ld = _rows(X)
    _check(lib().ml2_score_validity(v.handle, xp, n, ld, _ptr(valid_out), _ptr(margin_out),
                                    _stream(stream)))


def ml2_score_perf(p: Ensemble, X, valid, score_out, stream=None) -> None:
    xp, n, ld = _rows(X)
    _check(lib().ml2_score_perf(p.handle, xp, n, ld, _ptr(valid), _ptr(score_out),
                                _stream(stream)))


def ml2_score(v: Ensemble, p: Ensemble, X, valid_out, margin_out, score_out,
              stream=None) -> None:
    """Validity and performance in one call (one pass over the pool where
    the ensembles allow it)."""
    xp, n, ld = _rows(X)
    _check(lib().ml2_score(v.handle, p.handle, xp, n, ld, _ptr(valid_out), _ptr(margin_out),
                           _ptr(score_out), _stream(stream)))


def ml2_score_single_pass(v: Ensemble, p: Ensemble, X) -> bool:
    xp, n, ld = _rows(X)
    return bool(lib().ml2_score_single_pass(v.handle, p.handle, xp, n, ld))


def ml2_topk_workspace_bytes(n: int, k: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().ml2_topk_workspace_bytes(n, k, ctypes.byref(out)))
    return int(out.value)


def ml2_filter_topk(valid, scores, k: int, topk_idx, topk_score, num_selected, workspace,
                    workspace_bytes: int | None = None, n: int | None = None,
                    stream=None) -> None:
    if n is None:
        n = scores.shape[0]
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(lib().ml2_filter_topk(_ptr(valid), _ptr(scores), n, k, _ptr(topk_idx),
                                 _ptr(topk_score), _ptr(num_selected), _ptr(workspace),
                                 workspace_bytes, _stream(stream)))


def ml2_filter_topk_noalloc(valid, scores, k: int, topk_idx, topk_score, num_selected,
                            n: int | None = None, stream=None) -> None:
    """ml2_filter_topk with the library's static workspace (allocates nothing)."""
    if n is None:
        n = scores.shape[0]
    _check(lib().ml2_filter_topk_noalloc(_ptr(valid), _ptr(scores), n, k, _ptr(topk_idx),
                                         _ptr(topk_score), _ptr(num_selected), _stream(stream)))


def ml2_rerank_workspace_bytes(a: Ensemble, m: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().ml2_rerank_workspace_bytes(a.handle, m, ctypes.byref(out)))
    return int(out.value)


def ml2_rerank(a: Ensemble, X, rows, keep: int, row_scores, out_idx, out_score, num_selected,
               workspace, workspace_bytes: int | None = None, m: int | None = None,
               stream=None) -> None:
    xp, n, ld = _rows(X)
    if m is None:
        m = rows.shape[0]
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    _check(lib().ml2_rerank(a.handle, xp, n, ld, _ptr(rows), m, keep, _ptr(row_scores),
                            _ptr(out_idx), _ptr(out_score), _ptr(num_selected), _ptr(workspace),
                            workspace_bytes, _stream(stream)))


class Explorer:
    """An ml2_explorer over one pool of n candidates (owns the handle; holds
    references to its ensembles so they outlive it)."""

    def __init__(self, v: Ensemble, p: Ensemble, a: Ensemble | None, n: int, k: int,
                 keep: int, max_rounds: int):
        h = ctypes.c_void_p()
        _check(lib().ml2_explorer_create(v.handle, p.handle, a.handle if a else None, n, k, keep,
                                         max_rounds, ctypes.byref(h)))
        self.handle = h.value
        self.models = (v, p, a)
        self.n, self.k, self.keep = n, k, keep

    @property
    def rounds(self) -> int:
        return lib().ml2_explorer_rounds(self.handle)

    def reset(self) -> None:
        _check(lib().ml2_explorer_reset(self.handle))

    def round(self, X, out_idx, out_score, num_selected, rescore: bool = True,
              stream=None) -> None:
        xp, n, ld = _rows(X)
        if n != self.n:
            raise ValueError(f"pool has {n} rows, the explorer was made for {self.n}")
        _check(lib().ml2_explorer_round(self.handle, xp, ld, 1 if rescore else 0, _ptr(out_idx),
                                        _ptr(out_score), _ptr(num_selected), _stream(stream)))

    def free(self) -> None:
        if self.handle:
            lib().ml2_explorer_free(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover - interpreter shutdown order
        try:
            self.free()
        except Exception:
            pass


class StreamExplorer:
    """An ml2_stream_explorer: the explorer's rounds over a pool that arrives
    in chunks of rows (owns the handle; holds references to its ensembles)."""

    def __init__(self, v: Ensemble, p: Ensemble, a: Ensemble | None, max_chunk_rows: int,
                 k: int, keep: int, max_rounds: int):
        h = ctypes.c_void_p()
        _check(lib().ml2_stream_explorer_create(v.handle, p.handle, a.handle if a else None,
                                                max_chunk_rows, k, keep, max_rounds,
                                                ctypes.byref(h)))
        self.handle = h.value
        self.models = (v, p, a)
        self.k, self.keep = k, keep

    @property
    def rounds(self) -> int:
        return lib().ml2_stream_explorer_rounds(self.handle)

    def reset(self) -> None:
        _check(lib().ml2_stream_explorer_reset(self.handle))

    def begin(self, stream=None) -> None:
        _check(lib().ml2_stream_explorer_begin(self.handle, _stream(stream)))

    def chunk(self, X, row0: int, stream=None) -> None:
        xp, m, ld = _rows(X)
        _check(lib().ml2_stream_explorer_chunk(self.handle, xp, m, ld, row0, _stream(stream)))

    def end(self, out_idx, out_score, num_selected, stream=None) -> None:
        _check(lib().ml2_stream_explorer_end(self.handle, _ptr(out_idx), _ptr(out_score),
                                             _ptr(num_selected), _stream(stream)))

    def free(self) -> None:
        if self.handle:
            lib().ml2_stream_explorer_free(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover - interpreter shutdown order
        try:
            self.free()
        except Exception:
            pass


class Pipeline:
    """Device buffers for validity -> masked performance -> top-k on one pool
    (plumbing around the three calls; every step runs in libml2.so)."""

    def __init__(self, v: Ensemble, p: Ensemble, n: int, k: int, device="cuda",
                 with_margin: bool = False):
        import torch
        self.v, self.p, self.n, self.k = v, p, n, k
        self.valid = torch.empty(n, dtype=torch.uint8, device=device)
        self.margin = torch.empty(n, dtype=torch.float32, device=device) if with_margin else None
        self.score = torch.empty(n, dtype=torch.float32, device=device)
        self.idx = torch.empty(max(k, 1), dtype=torch.int32, device=device)
        self.top = torch.empty(max(k, 1), dtype=torch.float32, device=device)
        self.num = torch.empty(1, dtype=torch.int32, device=device)
        self.ws_bytes = ml2_topk_workspace_bytes(n, k)
        # 256-byte alignment holds for torch's caching allocator blocks
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        if self.ws.data_ptr() % 256:
            raise RuntimeError("top-k workspace is not 256-byte aligned")

    def run(self, X, stream=None) -> None:
        ml2_score_validity(self.v, X, self.valid, self.margin, stream)
        ml2_score_perf(self.p, X, self.valid, self.score, stream)
        ml2_filter_topk(self.valid, self.score, self.k, self.idx, self.top, self.num, self.ws,
                        self.ws_bytes, self.n, stream)


# ---- drawing from scores, and learning from what was drawn -----------------

class _Types:
    """torch's types that the operators take (torch is imported on first use)."""

    def __init__(self):
        import torch
        self.f32, self.i32 = torch.float32, torch.int32
        self.mask = (torch.uint8, torch.bool)
        self.code = {torch.float32: ML2_F32, torch.bfloat16: ML2_BF16, torch.float16: ML2_F16}
        self.current = torch._C._cuda_getDevice
        self.stream = torch._C._cuda_getCurrentRawStream


_types = None


def _t() -> _Types:
    global _types
    if _types is None:
        _types = _Types()
    return _types


def _dtype(t) -> int:
    d = _t().code.get(t)
    if d is None:
        raise ValueError(f"float32, bfloat16 or float16 expected, not {t}")
    return d


def _device(x, name: str) -> None:
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")


def _matrix(x, name: str):
    """(pointer, rows, columns, row stride) of a 2-D device tensor whose
    columns are contiguous; a single row may have any row stride."""
    _device(x, name)
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be a 2-D tensor with unit column stride")
    (rows, n), (ld, step) = shape, x.stride()
    if step != 1 and rows > 0 and n > 1:
        raise ValueError(f"{name} must be a 2-D tensor with unit column stride")
    return x.data_ptr(), rows, n, ld if rows > 1 and n > 0 else max(ld, n)


def _flat(x, name: str, dtype, shape):
    """Pointer of a contiguous device tensor of the given type and shape (or None)."""
    if x is None:
        return None
    if x.dtype is not dtype or x.shape != shape or not x.is_contiguous() or not x.is_cuda:
        raise ValueError(f"{name} must be a contiguous {dtype} device tensor of shape "
                         f"{tuple(shape)}")
    return x.data_ptr()


def _mask(valid, rows: int, n: int):
    """(pointer, row stride) of a uint8 mask [n] (shared) or [rows][n], or None."""
    if valid is None:
        return None, 0
    if valid.dtype not in _t().mask:
        raise ValueError("valid must be a uint8 or bool tensor")
    _device(valid, "valid")
    if valid.dim() == 1:
        if valid.shape[0] != n or (n > 1 and valid.stride(0) != 1):
            raise ValueError(f"valid must hold {n} contiguous entries")
        return valid.data_ptr(), 0
    p, r, c, ld = _matrix(valid, "valid")
    if (r, c) != (rows, n):
        raise ValueError(f"valid must be [{n}] or [{rows}][{n}]")
    return p, ld


def _on(device: str | None):
    import torch
    return torch.device("cuda") if device is None else torch.device(device)


def _space(ws):
    """(pointer, bytes) of a workspace tensor."""
    _device(ws, "workspace")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _workspace(size: int, device):
    import torch
    ws = torch.empty(max(size, 256), dtype=torch.uint8, device=device)
    if ws.data_ptr() % 256:  # holds for torch's caching allocator blocks
        raise RuntimeError("workspace is not 256-byte aligned")
    return ws


def _bytes(fn, *sizes) -> int:
    out = ctypes.c_size_t()
    _check(fn(*sizes, ctypes.byref(out)))
    return int(out.value)


def ml2_sample_workspace_bytes(n: int, rows: int, draws: int) -> int:
    return _bytes(lib().ml2_sample_workspace_bytes, n, rows, draws)


def ml2_sample(scores, u, idx, logprob, workspace, valid=None, temperature=None, top_k=None,
               top_p=None, min_p=None, stream=None) -> None:
    """Draws from each row of scores [rows][n] with given uniforms u [rows][draws]."""
    sp, rows, n, ld = _matrix(scores, "scores")
    draws = u.shape[-1]
    vp, vld = _mask(valid, rows, n)
    _check(lib().ml2_sample(
        _dtype(scores.dtype), sp, n, ld, rows, vp, vld,
        _flat(temperature, "temperature", _t().f32, (rows,)),
        _flat(top_k, "top_k", _t().i32, (rows,)), _flat(top_p, "top_p", _t().f32, (rows,)),
        _flat(min_p, "min_p", _t().f32, (rows,)), _flat(u, "u", _t().f32, (rows, draws)), draws,
        _flat(idx, "idx", _t().i32, (rows, draws)),
        _flat(logprob, "logprob", _t().f32, (rows, draws)), *_space(workspace),
        _stream(stream)))


def ml2_logprob_workspace_bytes(n: int, rows: int, per_row: int) -> int:
    return _bytes(lib().ml2_logprob_workspace_bytes, n, rows, per_row)


def ml2_logprob(scores, targets, logprob, workspace, valid=None, temperature=None,
                stream=None) -> None:
    """Log-probabilities of targets [rows][per_row] under each row's masked softmax."""
    sp, rows, n, ld = _matrix(scores, "scores")
    shape = (rows, targets.shape[-1])
    vp, vld = _mask(valid, rows, n)
    _check(lib().ml2_logprob(
        _dtype(scores.dtype), sp, n, ld, rows, vp, vld,
        _flat(temperature, "temperature", _t().f32, (rows,)),
        _flat(targets, "targets", _t().i32, shape), shape[1],
        _flat(logprob, "logprob", _t().f32, shape), *_space(workspace),
        _stream(stream)))


def ml2_logprob_grad(scores, targets, weight, grad, workspace, logprob=None, valid=None,
                     temperature=None, stream=None) -> None:
    """The gradient of sum_j weight_j * logprob_j to the scores, in their type
    (and the log-probabilities, where `logprob` is given)."""
    sp, rows, n, ld = _matrix(scores, "scores")
    gp, grows, gn, gld = _matrix(grad, "grad")
    if (grows, gn) != (rows, n) or grad.dtype != scores.dtype:
        raise ValueError("grad must have the shape and type of scores")
    shape = (rows, targets.shape[-1])
    vp, vld = _mask(valid, rows, n)
    _check(lib().ml2_logprob_grad(
        _dtype(scores.dtype), sp, n, ld, rows, vp, vld,
        _flat(temperature, "temperature", _t().f32, (rows,)),
        _flat(targets, "targets", _t().i32, shape), _flat(weight, "weight", _t().f32, shape),
        shape[1], _flat(logprob, "logprob", _t().f32, shape), gp, gld, *_space(workspace),
        _stream(stream)))


def ml2_embed(table, ids, out, scale: float = 1.0, stream=None) -> None:
    """out[i] = scale * table[ids[i]], zeros where ids[i] lies outside the table."""
    tp, V, D, ld = _matrix(table, "table")
    op, N, width, out_ld = _matrix(out, "out")
    if width != D or out.dtype != table.dtype:
        raise ValueError("out must have the table's width and type")
    _check(lib().ml2_embed(_dtype(table.dtype), tp, V, D, ld, _flat(ids, "ids", _t().i32, (N,)), N,
                           scale, op, out_ld, _stream(stream)))


def ml2_embed_grad_workspace_bytes(n: int, table_rows: int, width: int) -> int:
    return _bytes(lib().ml2_embed_grad_workspace_bytes, n, table_rows, width)


def ml2_embed_grad(dout, ids, grad, workspace, scale: float = 1.0, stream=None) -> None:
    """grad[v] = scale * sum of dout[i] over ids[i] == v, for every row of grad
    (float32 or dout's type)."""
    dp, N, D, ld = _matrix(dout, "dout")
    gp, V, width, gld = _matrix(grad, "grad")
    if width != D:
        raise ValueError("grad must have dout's width")
    _check(lib().ml2_embed_grad(_dtype(dout.dtype), dp, N, D, ld, _flat(ids, "ids", _t().i32, (N,)),
                                scale, _dtype(grad.dtype), gp, V, gld, *_space(workspace),
                                _stream(stream)))


class Sampler:
    """Buffers of ml2_sample for rows of n scores and `draws` draws a row."""

    def __init__(self, rows: int, n: int, draws: int = 1, device=None):
        import torch
        device = _on(device)
        self.idx = torch.empty(rows, draws, dtype=torch.int32, device=device)
        self.logprob = torch.empty(rows, draws, dtype=torch.float32, device=device)
        self.ws = _workspace(ml2_sample_workspace_bytes(n, rows, draws), device)

    def run(self, scores, u, valid=None, temperature=None, top_k=None, top_p=None, min_p=None,
            stream=None):
        """(idx, logprob), both [rows][draws]: this sampler's own buffers."""
        ml2_sample(scores, u, self.idx, self.logprob, self.ws, valid, temperature, top_k, top_p,
                   min_p, stream)
        return self.idx, self.logprob


class LogProb:
    """Buffers of ml2_logprob, and of ml2_logprob_grad where grad_dtype (the
    scores' type) is given, for rows of n scores and per_row targets a row."""

    def __init__(self, rows: int, n: int, per_row: int = 1, grad_dtype=None, device=None):
        import torch
        device = _on(device)
        self.logprob = torch.empty(rows, per_row, dtype=torch.float32, device=device)
        self.grad = None
        if grad_dtype is not None:
            self.grad = torch.empty(rows, n, dtype=grad_dtype, device=device)
        self.ws = _workspace(ml2_logprob_workspace_bytes(n, rows, per_row), device)

    def run(self, scores, targets, valid=None, temperature=None, stream=None):
        """logprob [rows][per_row]: this object's own buffer."""
        ml2_logprob(scores, targets, self.logprob, self.ws, valid, temperature, stream)
        return self.logprob

    def run_grad(self, scores, targets, weight, valid=None, temperature=None, stream=None):
        """(logprob, grad): this object's own buffers."""
        if self.grad is None:
            raise ValueError("made without grad_dtype")
        ml2_logprob_grad(scores, targets, weight, self.grad, self.ws, self.logprob, valid,
                         temperature, stream)
        return self.logprob, self.grad


class Embedding:
    """The output buffer of ml2_embed for n tokens of a table of one width."""

    def __init__(self, n: int, width: int, dtype, device=None):
        import torch
        self.out = torch.empty(n, width, dtype=dtype, device=_on(device))

    def run(self, table, ids, scale: float = 1.0, stream=None):
        """out [n][width]: this object's own buffer."""
        ml2_embed(table, ids, self.out, scale, stream)
        return self.out


class EmbeddingGrad:
    """Buffers of ml2_embed_grad: the gradient [table_rows][width] in grad_dtype
    for n tokens."""

    def __init__(self, n: int, table_rows: int, width: int, grad_dtype, device=None):
        import torch
        device = _on(device)
        self.grad = torch.empty(table_rows, width, dtype=grad_dtype, device=device)
        self.ws = _workspace(ml2_embed_grad_workspace_bytes(n, table_rows, width), device)

    def run(self, dout, ids, scale: float = 1.0, stream=None):
        """grad [table_rows][width]: this object's own buffer."""
        ml2_embed_grad(dout, ids, self.grad, self.ws, scale, stream)
        return self.grad


# ---- a training step: normalisation, gradient norms, the optimizer ----------

def _here(stream, *xs):
    """The stream of a call over these tensors (None among them): the current device's, on which
    they all have to be."""
    t = _t()
    at = t.current()
    for x in xs:
        if x is not None and x.get_device() != at:
            raise ValueError(f"tensors on device {x.get_device()}, the current one is {at}")
    return t.stream(at) if stream is None else _stream(stream)


def _param(x, name: str, dtype, width: int):
    """(pointer, type) of a parameter [width] of a row type or float32, or (None, the row type)."""
    if x is None:
        return None, _dtype(dtype)
    if x.dtype is not dtype and x.dtype is not _t().f32:
        raise ValueError(f"{name} must be {dtype} or float32, not {x.dtype}")
    return _flat(x, name, x.dtype, (width,)), _dtype(x.dtype)


def _same_type(a, b, names: str):
    """The type of two parameters of which each may be None."""
    if a is not None and b is not None and a.dtype is not b.dtype:
        raise ValueError(f"{names} must have one type")
    return a if a is not None else b


def ml2_layer_norm(x, weight, bias, out, mean=None, rstd=None, eps: float = 1e-5,
                   stream=None) -> None:
    """Layer norm of every row of x [rows][width]; weight and bias may be None."""
    xp, rows, width, ld = _matrix(x, "x")
    op, orows, owidth, out_ld = _matrix(out, "out")
    if (orows, owidth) != (rows, width) or out.dtype is not x.dtype:
        raise ValueError("out must have the shape and type of x")
    _same_type(weight, bias, "weight and bias")
    wp, code = _param(weight, "weight", x.dtype, width)
    bp, bcode = _param(bias, "bias", x.dtype, width)
    f32 = _t().f32
    _check(lib().ml2_layer_norm(_dtype(x.dtype), xp, rows, width, ld, bcode if wp is None else code,
                                wp, bp, eps, op, out_ld, _flat(mean, "mean", f32, (rows,)),
                                _flat(rstd, "rstd", f32, (rows,)),
                                _here(stream, x, weight, bias, out, mean, rstd)))


def ml2_layer_norm_grad_workspace_bytes(rows: int, width: int) -> int:
    return _bytes(lib().ml2_layer_norm_grad_workspace_bytes, rows, width)


def ml2_layer_norm_grad(x, dout, weight, mean, rstd, workspace, dx=None, dweight=None, dbias=None,
                        stream=None) -> None:
    """The gradients of ml2_layer_norm to its rows, weight and bias (each may be None)."""
    xp, rows, width, ld = _matrix(x, "x")
    dp, drows, dwidth, dout_ld = _matrix(dout, "dout")
    if (drows, dwidth) != (rows, width) or dout.dtype is not x.dtype:
        raise ValueError("dout must have the shape and type of x")
    dxp, dx_ld = None, width
    if dx is not None:
        dxp, r, w, dx_ld = _matrix(dx, "dx")
        if (r, w) != (rows, width) or dx.dtype is not x.dtype:
            raise ValueError("dx must have the shape and type of x")
    wp, code = _param(weight, "weight", x.dtype, width)
    _same_type(dweight, dbias, "dweight and dbias")
    gwp, gcode = _param(dweight, "dweight", x.dtype, width)
    gbp, bcode = _param(dbias, "dbias", x.dtype, width)
    f32 = _t().f32
    _check(lib().ml2_layer_norm_grad(
        _dtype(x.dtype), xp, rows, width, ld, dp, dout_ld, code, wp,
        _flat(mean, "mean", f32, (rows,)), _flat(rstd, "rstd", f32, (rows,)), dxp, dx_ld,
        bcode if gwp is None else gcode, gwp, gbp, *_space(workspace),
        _here(stream, x, dout, weight, mean, rstd, dx, dweight, dbias, workspace)))


def _tensors(xs, name: str):
    """The type of a list of contiguous device tensors of one type."""
    xs = list(xs)
    if not xs:
        raise ValueError(f"{name} must hold a tensor")
    for x in xs:
        if x is None or not x.is_cuda or not x.is_contiguous() or x.dtype is not xs[0].dtype:
            raise ValueError(f"{name} must be contiguous device tensors of one type")
        if x.device != xs[0].device:
            raise ValueError(f"{name} must be on one device")
    return xs, xs[0].dtype


def _like(grads, old):
    """A list of gradients that can take the place of another."""
    grads, dtype = _tensors(grads, "grads")
    if dtype is not old[0].dtype or grads[0].device != old[0].device or (
            [g.numel() for g in grads] != [g.numel() for g in old]):
        raise ValueError("grads must have the type, sizes and device of those before")
    return grads


def ml2_grad_norm_workspace_bytes(sizes) -> int:
    array = (ctypes.c_int64 * len(sizes))(*sizes)
    return _bytes(lib().ml2_grad_norm_workspace_bytes, array, len(sizes))


def ml2_adamw_state_bytes(state_bits: int, n: int) -> int:
    return _bytes(lib().ml2_adamw_state_bytes, state_bits, n)


def ml2_grad_norm(grads, norm, factor, workspace, max_norm: float = float("inf"),
                  scale: float = 1.0, step=None, stream=None) -> None:
    """The norm of all gradients together, and what a step multiplies them by (norm and factor:
    float32 [1], either may be None; step: int32 [1], raised by one where the norm is finite)."""
    grads, dtype = _tensors(grads, "grads")
    n = len(grads)
    t = _t()
    _check(lib().ml2_grad_norm(
        _dtype(dtype), (ctypes.c_void_p * n)(*[g.data_ptr() for g in grads]),
        (ctypes.c_int64 * n)(*[g.numel() for g in grads]), n, scale, max_norm,
        _flat(norm, "norm", t.f32, (1,)), _flat(factor, "factor", t.f32, (1,)),
        _flat(step, "step", t.i32, (1,)), *_space(workspace),
        _here(stream, grads[0], norm, factor, step, workspace)))


def ml2_adamw(param_dtype, grad_dtype, state_bits: int, tensors, count: int,
              options: ml2_adamw_options, stream=None) -> None:
    """A step of AdamW over an array of ml2_adamw_tensor.  It holds addresses, as the options do, so
    that nothing here can tell whether they are the current device's, as they have to be."""
    _check(lib().ml2_adamw(_dtype(param_dtype), _dtype(grad_dtype), state_bits, tensors, count,
                           ctypes.byref(options), _stream(stream)))


class LayerNorm:
    """Buffers of ml2_layer_norm for rows of one width."""

    def __init__(self, rows: int, width: int, dtype, device=None):
        import torch
        device = _on(device)
        self.out = torch.empty(rows, width, dtype=dtype, device=device)
        self.mean = torch.empty(rows, dtype=torch.float32, device=device)
        self.rstd = torch.empty(rows, dtype=torch.float32, device=device)
        self.shape, self.dtype, self.code = (rows, width), dtype, _dtype(dtype)
        self.buffers = (self.out.data_ptr(), width, self.mean.data_ptr(), self.rstd.data_ptr())

    def run(self, x, weight=None, bias=None, eps: float = 1e-5, stream=None):
        """(out, mean, rstd): this object's own buffers."""
        xp, rows, width, ld = _matrix(x, "x")
        if (rows, width) != self.shape or x.dtype is not self.dtype:
            raise ValueError("x must have the rows, width and type that this object was made for")
        _same_type(weight, bias, "weight and bias")
        wp, code = _param(weight, "weight", self.dtype, width)
        bp, bcode = _param(bias, "bias", self.dtype, width)
        _check(lib().ml2_layer_norm(self.code, xp, rows, width, ld, bcode if wp is None else code,
                                    wp, bp, eps, *self.buffers,
                                    _here(stream, x, weight, bias, self.out)))
        return self.out, self.mean, self.rstd


class LayerNormGrad:
    """Buffers of ml2_layer_norm_grad for rows of one width: dx in the rows' type, dweight and
    dbias (without bias: None) in grad_dtype."""

    def __init__(self, rows: int, width: int, dtype, grad_dtype=None, bias: bool = True,
                 device=None):
        import torch
        device = _on(device)
        grad_dtype = dtype if grad_dtype is None else grad_dtype
        self.dx = torch.empty(rows, width, dtype=dtype, device=device)
        self.dweight = torch.empty(width, dtype=grad_dtype, device=device)
        self.dbias = torch.empty(width, dtype=grad_dtype, device=device) if bias else None
        self.ws = _workspace(ml2_layer_norm_grad_workspace_bytes(rows, width), device)
        self.shape, self.dtype, self.code = (rows, width), dtype, _dtype(dtype)
        self.buffers = (self.dx.data_ptr(), width, _dtype(grad_dtype), self.dweight.data_ptr(),
                        _ptr(self.dbias), *_space(self.ws))

    def run(self, x, dout, weight, mean, rstd, stream=None):
        """(dx, dweight, dbias): this object's own buffers."""
        xp, rows, width, ld = _matrix(x, "x")
        dp, drows, dwidth, dout_ld = _matrix(dout, "dout")
        if (rows, width) != self.shape or (drows, dwidth) != self.shape or (
                x.dtype is not self.dtype or dout.dtype is not self.dtype):
            raise ValueError("x and dout must have the rows, width and type that this object was "
                             "made for")
        wp, code = _param(weight, "weight", self.dtype, width)
        f32 = _t().f32
        _check(lib().ml2_layer_norm_grad(
            self.code, xp, rows, width, ld, dp, dout_ld, code, wp,
            _flat(mean, "mean", f32, (rows,)), _flat(rstd, "rstd", f32, (rows,)), *self.buffers,
            _here(stream, x, dout, weight, mean, rstd, self.dx)))
        return self.dx, self.dweight, self.dbias


class GradNorm:
    """ml2_grad_norm over a program's gradient buffers, which it keeps (take() names others): norm
    and factor are this object's own buffers, and step, where given, the program's counter."""

    def __init__(self, grads, max_norm: float = float("inf"), scale: float = 1.0, step=None):
        import torch
        self.grads, self.dtype = _tensors(grads, "grads")
        count, self.step = len(self.grads), step
        self.norm, self.factor = (torch.empty(1, dtype=torch.float32, device=self.grads[0].device)
                                  for _ in range(2))
        sizes = [g.numel() for g in self.grads]
        self.at = (ctypes.c_void_p * count)()
        self.ws = _workspace(ml2_grad_norm_workspace_bytes(sizes), self.norm.device)
        self.args = (_dtype(self.dtype), self.at, (ctypes.c_int64 * count)(*sizes), count, scale,
                     max_norm, self.norm.data_ptr(), self.factor.data_ptr(),
                     _flat(step, "step", torch.int32, (1,)), *_space(self.ws))
        self.take(self.grads)

    def take(self, grads) -> None:
        """Other gradients of the same sizes and type from now on."""
        self.grads = _like(grads, self.grads)
        for i, g in enumerate(self.grads):
            self.at[i] = g.data_ptr()

    def run(self, stream=None):
        """(norm, factor), both float32 [1]: this object's own buffers."""
        _check(lib().ml2_grad_norm(*self.args, _here(stream, self.norm, self.step)))
        return self.norm, self.factor


_WHOLE = (int, np.integer)
_NUMBER = (float, np.floating, *_WHOLE)


class AdamW:
    """ml2_adamw over a program's parameters and gradient buffers, which it keeps (take() names
    other gradients).

    state_bits 32 or 8; m and v: lists of states (by default zeros: adamw_state); copies: a list
    of tensors of the gradients' type that get the new parameters too; weight_decay: one, or one
    for each tensor.  out: lists of parameters, m and v that a step writes instead of the own ones,
    which then stay as they were until accept() exchanges the two; None: in place."""

    def __init__(self, params, grads, state_bits: int = 32, m=None, v=None, copies=None,
                 weight_decay=0.01, betas=(0.9, 0.999), eps: float = 1e-8, seed: int = 0,
                 out=None):
        import torch
        self.params, self.dtype = _tensors(params, "params")
        self.grads, self.grad_dtype = _tensors(grads, "grads")
        self.state_bits, self.count = state_bits, len(self.params)
        sizes = [p.numel() for p in self.params]
        device = self.params[0].device

        def states(xs, name):
            if xs is None:
                return [adamw_state(n, state_bits, device) for n in sizes]
            xs, dtype = _tensors(xs, name)
            want = torch.float32 if state_bits == 32 else torch.uint8
            need = sizes if state_bits == 32 else [
                -(-n // ML2_STATE_BLOCK) * (ML2_STATE_BLOCK + 4) for n in sizes]
            if dtype is not want or [x.numel() for x in xs] != need:
                raise ValueError(f"{name} must be {want} of adamw_state's sizes")
            return xs

        self.m, self.v = states(m, "m"), states(v, "v")
        self.copies = None if copies is None else _tensors(copies, "copies")[0]
        self.out = None
        if out is not None:
            self.out = (_tensors(out[0], "params of out")[0], states(out[1], "m of out"),
                        states(out[2], "v of out"))
        if self.copies is not None and self.copies[0].dtype is not self.grad_dtype:
            raise ValueError("copies must have the gradients' type")
        if self.out is not None and self.out[0][0].dtype is not self.dtype:
            raise ValueError("params of out must have the parameters' type")
        for xs in (self.grads, self.copies, self.out and self.out[0]):
            if xs is not None and [x.numel() for x in xs] != sizes:
                raise ValueError("grads, copies and out must have the parameters' sizes")
        for xs in (self.grads, self.copies, self.m, self.v, *(self.out or ())):
            if xs is not None and xs[0].device != device:
                raise ValueError("all tensors must be on one device")
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else (
            [weight_decay] * self.count)
        if len(decay) != self.count:
            raise ValueError("weight_decay must be one number, or one for each tensor")
        self.options = ml2_adamw_options(0.0, betas[0], betas[1], eps, 1, None, None, None, seed)
        self.tensors = (ml2_adamw_tensor * self.count)()
        for t, n, d in zip(self.tensors, sizes, decay):
            t.n, t.weight_decay = n, d
        self._fill()

    def _fill(self) -> None:
        lists = (self.params, self.grads, self.m, self.v,
                 *(self.out or (self.params, self.m, self.v)))
        at = [[x.data_ptr() for x in xs] for xs in lists]
        copies = [x.data_ptr() for x in self.copies] if self.copies is not None else (
            [None] * self.count)
        for t, *t7, copy in zip(self.tensors, *at, copies):
            t.param, t.grad, t.m, t.v, t.param_out, t.m_out, t.v_out = t7
            t.copy = copy

    def take(self, grads) -> None:
        """Other gradients of the same sizes and type from now on."""
        self.grads = _like(grads, self.grads)
        self._fill()

    def accept(self) -> None:
        """The last step's results become the state, and the old state's memory the next
        step's output (without `out` the step was in place)."""
        if self.out is not None:
            old = (self.params, self.m, self.v)
            (self.params, self.m, self.v), self.out = self.out, old
            self._fill()

    def run(self, lr, step, factor=None, stream=None):
        """The new parameters.  lr: a number, or float32 [1] on the device; step: a whole number, or
        int32 [1] on the device; factor: float32 [1] on the device, as GradNorm's, or None."""
        if lr is None or step is None:  # _flat() lets None pass, and the last call's would stay
            raise ValueError("lr and step must be given")
        o, t = self.options, _t()
        o.lr_device = o.step_device = None
        used = [self.params[0], factor]
        if isinstance(lr, _NUMBER):
            o.lr = lr
        else:
            o.lr_device = _flat(lr, "lr", t.f32, (1,))
            used.append(lr)
        if isinstance(step, _WHOLE):
            o.step = int(step)
        else:
            o.step_device = _flat(step, "step", t.i32, (1,))
            used.append(step)
        o.factor = _flat(factor, "factor", t.f32, (1,))
        ml2_adamw(self.dtype, self.grad_dtype, self.state_bits, self.tensors, self.count, o,
                  _here(stream, *used))
        return self.out[0] if self.out is not None else self.params


def adamw_state(n: int, state_bits: int = 32, device=None):
    """A state of zeros for n elements: float32 [n], or the bytes of an 8-bit state."""
    import torch
    dtype = torch.float32 if state_bits == 32 else torch.uint8
    size = ml2_adamw_state_bytes(state_bits, n) // dtype.itemsize
    return torch.zeros(size, dtype=dtype, device=_on(device))


def adamw_state_parts(state, n: int):
    """An 8-bit state's numbers (float8_e4m3fn [n], in units of their block's scale) and scales
    (float32, one for each ML2_STATE_BLOCK elements), as views."""
    import torch
    codes = -(-n // ML2_STATE_BLOCK) * ML2_STATE_BLOCK
    return state[:n].view(torch.float8_e4m3fn), state[codes:].view(torch.float32)


# ---- microbenchmarks (include/ml2_probe.h) ---------------------------------

def _probe(fn, *args):
    ms, work = ctypes.c_double(), ctypes.c_double()
    _check(fn(*args, ctypes.byref(ms), ctypes.byref(work)))
    return ms.value, work.value


def ml2_probe_visit(depth: int, trees_per_lane: int, lanes_per_candidate: int, waves: int,
                    features: int, iters: int, blocks: int):
    """(ms, node visits) of the walk's inner loop over a resident chunk at
    the given shape."""
    return _probe(lib().ml2_probe_visit, depth, trees_per_lane, lanes_per_candidate, waves,
                  features, iters, blocks)


def ml2_probe_lds(mode: int, iters: int, blocks: int):
    """(ms, bytes read) of LDS reads of 4/8/16 bytes (mode % 3), consecutive
    (mode < 3) or random."""
    return _probe(lib().ml2_probe_lds, mode, iters, blocks)


def ml2_probe_valu(iters: int, blocks: int):
    """(ms, lane additions) of chains of 32-bit adds."""
    return _probe(lib().ml2_probe_valu, iters, blocks)


# ---- tuning overrides (include/ml2_probe.h) --------------------------------

def ml2_tune_walk_plan(split: int = 0, group: int = 0, waves: int = 0, nbuf: int = 0,
                       chunk: int = 0) -> None:
    """Force the walks' launch shape for every later call (zeros: the
    planner's choice); results are unchanged, only the shape differs."""
    _check(lib().ml2_tune_walk_plan(split, group, waves, nbuf, chunk))


def ml2_tune_layout(layout: int = 0) -> None:
    """Force the layout of later loads: 0 the loader's choice, 1 perfect,
    2 ragged (where the ensemble allows it)."""
    _check(lib().ml2_tune_layout(layout))


def ml2_probe_walk(e: Ensemble, X, n: int, ld: int, perf: bool, masked: bool) -> ml2_walk_info:
    """The walk that ml2_score_validity (perf: ml2_score_perf, masked: with a
    mask) takes over n rows at X (a tensor or an address) with row stride ld."""
    info = ml2_walk_info()
    _check(lib().ml2_probe_walk(e.handle, _ptr(X), n, ld, int(perf), int(masked),
                                ctypes.byref(info)))
    return info
