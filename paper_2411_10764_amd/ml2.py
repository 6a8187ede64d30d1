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
                ("ml2_embed_grad", [I32, P, I64, I64, I64, P, F32, I32, P, I64, I64, P, SZ, P])):
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
