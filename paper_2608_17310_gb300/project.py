"""Python binding of the products whose rows choose their weights (``include/es_project.h``): a
projection with a low-rank adapter per request beside it, and the layer of experts, between
``es_perturb`` and ``es_restore``.

Argument marshalling only, as in ``esopt`` and ``rollout``: every function forwards to the
function of the same name in ``libesopt.so``. Arguments are torch CUDA tensors; errors are
``esopt.EsError``, or ``ValueError`` for tensors of the wrong type, shape or layout and numbers
that C's types do not hold.

    weights = pj.es_weights_create(w)                       # [out, in], or [experts, out, in]
    adapters = pj.es_adapters_create(a, b, scale)           # [members, rank, in], [members, out, rank]
    workspace = torch.zeros(pj.es_project_workspace(weights, rows, adapters), dtype=torch.uint8, device="cuda")
    pj.es_project(weights, x, y, workspace, adapters=adapters, adapter=member_of_request, start=start)

    pj.es_route(scores, chosen, weight, start, rows, places, route_workspace)
    pj.es_project_experts(up, x, h, start, workspace, rows=rows, gated=True)
    pj.es_project_experts(down, h, z, start, workspace)
    pj.es_combine(z, places, weight, out, add=x)
"""
from __future__ import annotations

import ctypes
from struct import Struct, error as _StructError

from . import esopt, rollout
from .esopt import ES_BF16, ES_FP32, ES_FP8_E4M3, EsError, _check  # noqa: F401
from .rollout import _stream, _tensor

ES_MAX_EXPERTS = 1024
ES_MAX_ROWS = 16777216
ES_PROJECT_GAVE_UP = 4096

_VP, _U64, _INT = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int


class es_weights_desc_t(ctypes.Structure):
    _fields_ = [("data", _VP), ("scale", _VP), ("group_stride", _U64), ("row_stride", _U64), ("groups", _INT),
                ("out_features", _INT), ("in_features", _INT), ("dtype", _INT)]


class es_adapters_desc_t(ctypes.Structure):
    _fields_ = [("a", _VP), ("b", _VP), ("scale", _VP), ("a_stride", _U64), ("b_stride", _U64), ("count", _INT),
                ("rank", _INT), ("out_features", _INT), ("in_features", _INT)]


class es_project_t(ctypes.Structure):
    _fields_ = [("x", _VP), ("y", _VP), ("start", _VP), ("adapter", _VP), ("x_stride", _U64), ("y_stride", _U64),
                ("rows", _INT), ("requests", _INT)]


class es_project_experts_t(ctypes.Structure):
    _fields_ = [("x", _VP), ("y", _VP), ("start", _VP), ("rows", _VP), ("x_stride", _U64), ("y_stride", _U64),
                ("x_rows", _INT), ("slots", _INT), ("gated", _INT)]


class es_route_t(ctypes.Structure):
    _fields_ = [("scores", _VP), ("chosen", _VP), ("weights", _VP), ("start", _VP), ("rows", _VP), ("places", _VP),
                ("scores_stride", _U64), ("tokens", _INT), ("experts", _INT), ("top", _INT), ("normalise", _INT),
                ("dtype", _INT)]


class es_combine_t(ctypes.Structure):
    _fields_ = [("y", _VP), ("places", _VP), ("weights", _VP), ("add", _VP), ("out", _VP), ("y_stride", _U64),
                ("add_stride", _U64), ("out_stride", _U64), ("slots", _INT), ("tokens", _INT), ("top", _INT),
                ("features", _INT)]


# Small calls are bound by their host time: arguments are packed as bytes (rollout says why).
_PROJECT = Struct("6Q2i")
_EXPERTS = Struct("6Q3i4x")
_ROUTE = Struct("7Q5i4x")
_COMBINE = Struct("8Q4i")
for _packed, _structure in ((_PROJECT, es_project_t), (_EXPERTS, es_project_experts_t), (_ROUTE, es_route_t),
                            (_COMBINE, es_combine_t)):
    assert _packed.size == ctypes.sizeof(_structure)

_calls = None
_BF16 = _F32 = _I32 = _U8 = None


def _lib() -> ctypes.CDLL:
    global _calls, _BF16, _F32, _I32, _U8
    if _calls is None:
        import torch
        _BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
        rollout._lib()
        L = esopt.lib()
        P = ctypes.POINTER
        for name, res, args in (
                ("es_weights_create", _INT, [P(es_weights_desc_t), P(_VP)]),
                ("es_weights_destroy", _INT, [_VP]),
                ("es_adapters_create", _INT, [P(es_adapters_desc_t), P(_VP)]),
                ("es_adapters_destroy", _INT, [_VP]),
                ("es_project_workspace", _U64, [_VP, _VP, _INT]),
                ("es_project", _INT, [_VP, _VP, _VP, _VP, _U64, _VP]),
                ("es_project_experts", _INT, [_VP, _VP, _VP, _U64, _VP]),
                ("es_route_workspace", _U64, [_INT, _INT, _INT]),
                ("es_route", _INT, [_VP, _VP, _U64, _VP]),
                ("es_combine", _INT, [_VP, _VP])):
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _calls = L
    return _calls


def _matrix(t, what: str, rows=None, width=None):
    """Address, row stride, rows and width of a bfloat16 matrix whose rows are contiguous."""
    if t.dtype is not _BF16 or not t.is_cuda:
        raise ValueError(f"{what} must be a bfloat16 CUDA tensor")
    shape = t.shape
    if len(shape) == 2 and (rows is None or shape[0] == rows) and (width is None or shape[1] == width):
        if t.is_contiguous():
            return t.data_ptr(), shape[1], shape[0], shape[1]
        stride = t.stride()
        if stride[1] == 1:
            # torch gives a single row any stride; what it is does not matter then
            return t.data_ptr(), stride[0] if shape[0] > 1 else shape[1], shape[0], shape[1]
    raise ValueError(f"{what} must be {'some' if rows is None else rows} contiguous rows of {'some' if width is None else width}, got "
                     f"shape {tuple(shape)} with strides {t.stride()}")


def _pack(layout, call, *args):
    try:
        return layout.pack(*args)
    except (_StructError, OverflowError) as e:
        raise ValueError(f"{call}: {e}") from None


class _Handle:
    _destroy = ""

    def __init__(self, handle, keepalive):
        self.handle = handle
        self._keepalive = keepalive

    def close(self) -> None:
        if self.handle:
            h, self.handle = self.handle, None
            _check(getattr(_lib(), self._destroy)(h), self._destroy)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class Weights(_Handle):
    """Owns an ``es_weights_t``. Keeps the matrices' tensors alive."""
    _destroy = "es_weights_destroy"


class Adapters(_Handle):
    """Owns an ``es_adapters_t``. Keeps the adapters' tensors alive."""
    _destroy = "es_adapters_destroy"


def es_weights_create(w, scale=None) -> Weights:
    """Matrices [out, in] or [groups, out, in] of bfloat16, or of E4M3 codes (float8_e4m3fn or
    uint8) with float32 scales [groups] (one matrix: any shape of one element). Rows are
    contiguous; rows and matrices may lie further apart."""
    import torch
    _lib()
    if w.dtype == torch.bfloat16:
        dtype = ES_BF16
    elif w.dtype in (torch.float8_e4m3fn, torch.uint8):
        dtype = ES_FP8_E4M3
    else:
        raise ValueError(f"matrices are bfloat16 or FP8 E4M3, not {w.dtype}")
    if w.dim() not in (2, 3) or not w.is_cuda:
        raise ValueError("w must be a CUDA tensor [out, in] or [groups, out, in]")
    v = w[None] if w.dim() == 2 else w
    groups, out, width = v.shape
    if width > 1 and v.stride(2) != 1:
        raise ValueError("w: rows must be contiguous")
    row = v.stride(1) if out > 1 else width
    d = es_weights_desc_t(v.data_ptr(), _tensor(scale, torch.float32, "scale", groups), v.stride(0) if groups > 1 else 0, row,
                          groups, out, width, dtype)
    handle = _VP()
    _check(_lib().es_weights_create(ctypes.byref(d), ctypes.byref(handle)), "es_weights_create")
    made = Weights(handle.value, (w, scale))
    made.groups, made.out_features, made.in_features = groups, out, width
    return made


def es_adapters_create(a, b, scale=None) -> Adapters:
    """Adapters of one projection: ``a`` [count, rank, in] and ``b`` [count, out, rank] of
    bfloat16, each matrix contiguous; ``scale`` float32 [count]."""
    import torch
    _lib()
    for t, what in ((a, "a"), (b, "b")):
        if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 3:
            raise ValueError(f"{what} must be a bfloat16 CUDA tensor of three axes")
        if t.shape[0] and not t[0].is_contiguous():
            raise ValueError(f"{what}: a matrix must be contiguous")
    count, rank, width = a.shape
    out = b.shape[1]
    if b.shape[0] != count or b.shape[2] != rank:
        raise ValueError(f"a {tuple(a.shape)} and b {tuple(b.shape)} do not go together")
    d = es_adapters_desc_t(a.data_ptr(), b.data_ptr(), _tensor(scale, torch.float32, "scale", count),
                           a.stride(0) if count > 1 else 0, b.stride(0) if count > 1 else 0, count, rank, out, width)
    handle = _VP()
    _check(_lib().es_adapters_create(ctypes.byref(d), ctypes.byref(handle)), "es_adapters_create")
    made = Adapters(handle.value, (a, b, scale))
    made.count, made.rank = count, rank
    return made


def _int(n, what: str) -> int:
    n = int(n)
    if not -2 ** 31 <= n < 2 ** 31:  # ctypes would cut it
        raise ValueError(f"{what} {n} must be a 32-bit number")
    return n


def es_project_workspace(weights: Weights, rows: int, adapters: Adapters = None) -> int:
    """Bytes of (zeroed) workspace for es_project, or es_project_experts, of up to ``rows`` rows.
    Without adapters and named rows ES_PROJECT_GAVE_UP + 256 bytes do."""
    return int(_lib().es_project_workspace(weights.handle, adapters.handle if adapters is not None else None, _int(rows, "rows")))


def es_project_gave_up(workspace) -> bool:
    """Whether a kernel that used this workspace gave up a wait (an error of the library): its
    outputs since are not to be used, nor the workspace before it has been zeroed. Waits for the
    current stream; a program asks where it reads results anyway."""
    return bool(workspace[ES_PROJECT_GAVE_UP:ES_PROJECT_GAVE_UP + 4].any())


def es_project(weights: Weights, x, y, workspace, adapters: Adapters = None, adapter=None, start=None, stream=None) -> None:
    """y = W x for rows ``x`` [rows, in], plus the adapter of each row's request: ``adapter`` int32
    [requests], ``start`` int32 [requests + 1] (None: one row each)."""
    x_ptr, x_stride, rows, _ = _matrix(x, "x", None, weights.in_features)
    y_ptr, y_stride, _, _ = _matrix(y, "y", rows, weights.out_features)
    requests = rows
    if adapter is not None:
        requests = adapter.numel()
    elif start is not None:
        requests = start.numel() - 1
    args = _pack(_PROJECT, "es_project", x_ptr, y_ptr, _tensor(start, _I32, "start", requests + 1),
                 _tensor(adapter, _I32, "adapter", requests), x_stride, y_stride, rows, requests)
    status = _calls.es_project(weights.handle, adapters.handle if adapters is not None else None, args,
                               _tensor(workspace, _U8, "workspace"), workspace.numel(), _stream(stream))
    if status:
        _check(status, "es_project")


def es_project_experts(weights: Weights, x, y, start, workspace, rows=None, gated: bool = False, stream=None) -> None:
    """Rows of ``y`` [slots, out] from start[g] to start[g + 1] - 1 are W_g times the rows of ``x``
    that ``rows`` (int32 [slots]) names, or times x's own; gated: silu of the product's first half
    times its second."""
    x_ptr, x_stride, x_rows, _ = _matrix(x, "x", None, weights.in_features)
    out = weights.out_features
    if gated and out % 2:
        raise ValueError(f"a gated product of {out} features")
    y_ptr, y_stride, slots, _ = _matrix(y, "y", None, out // 2 if gated else out)
    args = _pack(_EXPERTS, "es_project_experts", x_ptr, y_ptr, _tensor(start, _I32, "start", weights.groups + 1),
                 _tensor(rows, _I32, "rows", slots), x_stride, y_stride, x_rows, slots, bool(gated))
    status = _calls.es_project_experts(weights.handle, args, _tensor(workspace, _U8, "workspace"), workspace.numel(),
                                       _stream(stream))
    if status:
        _check(status, "es_project_experts")


def es_route_workspace(tokens: int, experts: int, top: int) -> int:
    """Bytes of workspace for es_route of up to ``tokens`` tokens."""
    return int(_lib().es_route_workspace(_int(tokens, "tokens"), _int(experts, "experts"), _int(top, "top")))


def es_route(scores, chosen, weights, start, rows, places, workspace, normalise: bool = True, stream=None) -> None:
    """The experts of each token of ``scores`` [tokens, experts] (bfloat16 or float32): ``chosen``
    int32 and ``weights`` float32 [tokens, top], and their order by expert: ``start`` int32
    [experts + 1], ``rows`` int32 [tokens * top], ``places`` int32 [tokens, top]."""
    _lib()
    if scores.dtype is _BF16:
        dtype = ES_BF16
    elif scores.dtype is _F32:
        dtype = ES_FP32
    else:
        raise ValueError(f"scores are bfloat16 or float32, not {scores.dtype}")
    if not scores.is_cuda or scores.dim() != 2 or (scores.shape[1] > 1 and scores.shape[0] and scores.stride(1) != 1):
        raise ValueError("scores must be a CUDA tensor of contiguous rows [tokens, experts]")
    tokens, experts = scores.shape
    if chosen.dim() != 2 or chosen.shape[0] != tokens:
        raise ValueError(f"chosen must be [{tokens}, top]")
    top = chosen.shape[1]
    n = tokens * top
    if weights.shape != chosen.shape or places.shape != chosen.shape:
        raise ValueError(f"weights and places must be {tuple(chosen.shape)}, as chosen is")
    args = _pack(_ROUTE, "es_route", scores.data_ptr(), _tensor(chosen, _I32, "chosen"), _tensor(weights, _F32, "weights"),
                 _tensor(start, _I32, "start", experts + 1), _tensor(rows, _I32, "rows", n), _tensor(places, _I32, "places"),
                 scores.stride(0) if tokens > 1 else experts, tokens, experts, top, bool(normalise), dtype)
    status = _calls.es_route(args, _tensor(workspace, _U8, "workspace"), workspace.numel(), _stream(stream))
    if status:
        _check(status, "es_route")


def es_combine(y, places, weights, out, add=None, stream=None) -> None:
    """out[t] = sum over j of weights[t, j] * y[places[t, j]], plus add[t]: bfloat16 rows ``y``
    [slots, features], ``out`` and ``add`` [tokens, features]; ``places`` int32 and ``weights``
    float32 [tokens, top]."""
    _lib()
    y_ptr, y_stride, slots, features = _matrix(y, "y")
    out_ptr, out_stride, tokens, _ = _matrix(out, "out", None, features)
    add_ptr = add_stride = 0
    if add is not None:
        add_ptr, add_stride, _, _ = _matrix(add, "add", tokens, features)
    if places.dim() != 2 or places.shape[0] != tokens or weights.shape != places.shape:
        raise ValueError(f"places and weights must be [{tokens}, top] alike")
    args = _pack(_COMBINE, "es_combine", y_ptr, _tensor(places, _I32, "places"), _tensor(weights, _F32, "weights"), add_ptr,
                 out_ptr, y_stride, add_stride, out_stride, slots, tokens, places.shape[1], features)
    status = _calls.es_combine(args, _stream(stream))
    if status:
        _check(status, "es_combine")
