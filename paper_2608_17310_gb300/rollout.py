"""Python binding of the rollout operators (``include/es_rollout.h``): a paged
key/value cache that is appended to, read back and attended over, between
``es_perturb`` and ``es_restore``.

Argument marshalling only, as in ``esopt``: every function forwards to the function
of the same name in ``libesopt.so``. Arguments are torch CUDA tensors (or their
device pointers, where a shape is not needed); errors are ``esopt.EsError``, or
``ValueError`` for tensors of the wrong type, shape or layout and numbers that C's types do
not hold.

    cache = ro.es_cache_create(k_pages, v_pages)            # [pages, kv_heads, page_size, head_dim]
    batch = ro.Batch(page_table, seq_len, start, tokens, max_new)
    ro.es_cache_append(cache, batch, qkv, q, q_norm, k_norm, rope)
    ro.es_attention(cache, batch, q, out, workspace, scale=head_dim ** -0.5)
"""
from __future__ import annotations

import ctypes
from struct import Struct, error as _StructError

from . import esopt
from .esopt import ES_BF16, ES_FP8_E4M3, EsError, _check  # noqa: F401

ES_MAX_SEQUENCES = 4096
ES_ATTENTION_GAVE_UP = 4096

_VP, _U64, _INT, _FLOAT = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int, ctypes.c_float


class es_cache_desc_t(ctypes.Structure):
    _fields_ = [("k", _VP), ("v", _VP), ("k_scale", _VP), ("v_scale", _VP), ("num_pages", _U64),
                ("page_stride", _U64), ("scale_stride", _U64), ("page_size", _INT),
                ("kv_heads", _INT), ("head_dim", _INT), ("dtype", _INT)]


class es_batch_t(ctypes.Structure):
    _fields_ = [("pages", _VP), ("seq_len", _VP), ("start", _VP), ("pages_per_row", _INT),
                ("sequences", _INT), ("tokens", _INT), ("max_new", _INT)]


class es_append_t(ctypes.Structure):
    _fields_ = [("qkv", _VP), ("q_out", _VP), ("q_weight", _VP), ("k_weight", _VP), ("rope", _VP),
                ("positions", _VP), ("qkv_stride", _U64), ("q_out_stride", _U64),
                ("rope_rows", _U64), ("q_heads", _INT), ("rotary_dim", _INT),
                ("interleaved", _INT), ("eps", _FLOAT)]


class es_attention_t(ctypes.Structure):
    _fields_ = [("q", _VP), ("out", _VP), ("lse", _VP), ("slopes", _VP), ("first", _VP),
                ("last", _VP), ("q_stride", _U64), ("out_stride", _U64), ("q_heads", _INT),
                ("window", _INT), ("scale", _FLOAT), ("softcap", _FLOAT)]


# Small calls are bound by their host time, so the functions pack es_append_t and
# es_attention_t as bytes (a ctypes structure takes 0.4 us more to make) and ask for the current
# stream's handle alone.
_APPEND = Struct("9Q3if")
_ATTENTION = Struct("8Q2i2f")
assert _APPEND.size == ctypes.sizeof(es_append_t) and _ATTENTION.size == ctypes.sizeof(es_attention_t)

_calls = None
_BF16 = _F32 = _I32 = _U8 = None  # torch's, once it is in use
_raw_stream = _device = None


def _lib() -> ctypes.CDLL:
    global _calls, _BF16, _F32, _I32, _U8, _raw_stream, _device
    if _calls is None:
        import torch
        _BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _device = getattr(torch._C, "_cuda_getDevice", None)
        L = esopt.lib()
        P = ctypes.POINTER
        for name, res, args in (
                ("es_cache_create", _INT, [P(es_cache_desc_t), P(_VP)]),
                ("es_cache_destroy", _INT, [_VP]),
                ("es_cache_append", _INT, [_VP, P(es_batch_t), _VP, _VP]),
                ("es_cache_read", _INT, [_VP, P(es_batch_t), _VP, _VP, _VP]),
                ("es_attention", _INT, [_VP, P(es_batch_t), _VP, _VP, _U64, _VP]),
                ("es_attention_workspace", _U64, [_VP, _INT])):
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _calls = L
    return _calls


def _stream(stream) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(_device())
    return esopt._stream(stream)


def _tensor(t, dtype, what: str, numel=None) -> int:
    """The address of a contiguous CUDA tensor of this dtype (and number of elements); None is
    NULL."""
    if t is None:
        return 0
    if t.dtype is not dtype or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{what} must be a contiguous CUDA tensor of {dtype}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, not {numel} elements")
    return t.data_ptr()


def _rows(t, rows: int, heads, head_dim: int, what: str):
    """Address, row stride and heads of bf16 rows [rows, heads, head_dim] or
    [rows, heads * head_dim] whose rows are contiguous; heads None: as many as there are."""
    if t.dtype is not _BF16 or not t.is_cuda:
        raise ValueError(f"{what} must be a bfloat16 CUDA tensor")
    shape = t.shape
    n = len(shape)
    if n == 3:
        have, fits = shape[1], shape[2] == head_dim
    elif n == 2:
        have, fits = divmod(shape[1], head_dim)
        fits = fits == 0
    else:
        have, fits = 0, False
    if fits and shape[0] == rows and (heads is None or heads == have):
        width = have * head_dim
        if rows == 0 or t.is_contiguous():
            return t.data_ptr(), width, have
        stride = t.stride()
        if stride[-1] == 1 and (n == 2 or have == 1 or stride[1] == head_dim):
            # torch gives a single row any stride; what it is does not matter then
            return t.data_ptr(), stride[0] if rows > 1 else width, have
    raise ValueError(f"{what} must be {rows} contiguous rows of {heads or 'some'} heads of {head_dim}, got "
                     f"shape {tuple(shape)} with strides {t.stride()}")


class Cache:
    """Owns an ``es_cache_t``. Keeps the page tensors alive."""

    def __init__(self, handle, desc, keepalive):
        self.handle = handle
        self.kv_heads, self.head_dim = desc.kv_heads, desc.head_dim
        self.page_size, self.dtype = desc.page_size, desc.dtype
        self._keepalive = keepalive

    def close(self) -> None:
        if self.handle:
            h, self.handle = self.handle, None
            _check(_lib().es_cache_destroy(h), "es_cache_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def es_cache_create(k, v, k_scale=None, v_scale=None) -> Cache:
    """A cache over page tensors [pages, kv_heads, page_size, head_dim] of bfloat16, or of
    E4M3 codes (float8_e4m3fn or uint8) with float32 scales [pages, kv_heads, page_size].
    Each page is contiguous; pages may lie further apart, alike in k and v."""
    import torch
    _lib()
    if k.dtype == torch.bfloat16:
        dtype = ES_BF16
    elif k.dtype in (torch.float8_e4m3fn, torch.uint8):
        dtype = ES_FP8_E4M3
    else:
        raise ValueError(f"a cache is bfloat16 or FP8 E4M3, not {k.dtype}")
    if v.dtype != k.dtype or v.shape != k.shape or k.dim() != 4:
        raise ValueError("k and v must be alike, [pages, kv_heads, page_size, head_dim]")

    def stride(t, what):
        if not t.is_cuda:
            raise ValueError(f"{what} must be a CUDA tensor")
        page = t[0] if t.shape[0] else t
        if t.shape[0] and not page.is_contiguous():
            raise ValueError(f"{what}: a page must be contiguous")
        return t.stride(0) if t.shape[0] > 1 else page.numel()

    page_stride = stride(k, "k")
    if stride(v, "v") != page_stride:
        raise ValueError("k and v pages lie at different strides")
    scale_stride = 0
    if (k_scale is None) != (v_scale is None):
        raise ValueError("k_scale and v_scale go together")
    if k_scale is not None:
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.dtype != torch.float32 or t.shape != k.shape[:3]:
                raise ValueError(f"{what} must be float32 {tuple(k.shape[:3])}")
        scale_stride = stride(k_scale, "k_scale")
        if stride(v_scale, "v_scale") != scale_stride:
            raise ValueError("k_scale and v_scale pages lie at different strides")
    d = es_cache_desc_t(k.data_ptr(), v.data_ptr(),
                        0 if k_scale is None else k_scale.data_ptr(),
                        0 if v_scale is None else v_scale.data_ptr(),
                        k.shape[0], page_stride, scale_stride, k.shape[2], k.shape[1], k.shape[3],
                        dtype)
    handle = _VP()
    _check(_lib().es_cache_create(ctypes.byref(d), ctypes.byref(handle)), "es_cache_create")
    return Cache(handle.value, d, (k, v, k_scale, v_scale))


class Batch:
    """The sequences of a call (``es_batch_t``): a page table [sequences, pages_per_row], the
    lengths [sequences] with the new tokens included, and where each sequence's new tokens
    begin [sequences + 1] (None: one each), all int32 CUDA tensors that the caller may
    rewrite between calls. ``tokens`` and ``max_new`` bound what ``start`` may hold then."""

    def __init__(self, pages, seq_len, start=None, tokens=None, max_new=None):
        _lib()
        if pages.dim() != 2:
            raise ValueError("pages must be [sequences, pages_per_row]")
        n = pages.shape[0]
        if tokens is None or max_new is None:
            if start is not None:
                raise ValueError("tokens and max_new go with start")
            tokens, max_new = n, 1
        self.tokens, max_new = int(tokens), int(max_new)
        if not (-2 ** 31 <= self.tokens < 2 ** 31 and -2 ** 31 <= max_new < 2 ** 31):  # ctypes would cut them
            raise ValueError(f"tokens {self.tokens} and max_new {max_new} must be 32-bit numbers")
        self._keepalive = (pages, seq_len, start)
        self.args = es_batch_t(_tensor(pages, _I32, "pages"),
                               _tensor(seq_len, _I32, "seq_len", n),
                               _tensor(start, _I32, "start", n + 1),
                               pages.shape[1], n, self.tokens, max_new)
        self.ref = ctypes.byref(self.args)


def es_cache_append(cache: Cache, batch: Batch, qkv, q_out, q_weight=None, k_weight=None,
                    rope=None, eps: float = 1e-6, positions=None, interleaved: bool = False,
                    stream=None) -> None:
    """Head norms, rotation and cache write of the batch's new tokens. ``rope``: float32
    [rows, rotary_dim / 2, 2] of (cos, sin)."""
    d, n = cache.head_dim, batch.tokens
    q_ptr, q_stride, q_heads = _rows(q_out, n, None, d, "q_out")
    x_ptr, x_stride, _ = _rows(qkv, n, q_heads + 2 * cache.kv_heads, d, "qkv")
    rope_ptr = rope_rows = rotary_dim = 0
    if rope is not None:
        shape = rope.shape
        if len(shape) != 3 or shape[2] != 2:
            raise ValueError("rope must be [rows, rotary_dim / 2, 2]")
        rope_ptr, rope_rows, rotary_dim = _tensor(rope, _F32, "rope"), shape[0], 2 * shape[1]
    try:
        args = _APPEND.pack(
            x_ptr, q_ptr, _tensor(q_weight, _BF16, "q_weight", d), _tensor(k_weight, _BF16, "k_weight", d),
            rope_ptr, _tensor(positions, _I32, "positions", n), x_stride, q_stride, rope_rows, q_heads,
            rotary_dim, interleaved, eps)
    except (_StructError, OverflowError) as e:
        raise ValueError(f"es_cache_append: {e}") from None
    status = _calls.es_cache_append(cache.handle, batch.ref, args, _stream(stream))
    if status:
        _check(status, "es_cache_append")


def es_cache_read(cache: Cache, batch: Batch, k_out=None, v_out=None, stream=None) -> None:
    """The cached keys and values of the batch's tokens as bfloat16
    [tokens, kv_heads, head_dim]."""
    shape = (batch.tokens, cache.kv_heads, cache.head_dim)
    for t, what in ((k_out, "k_out"), (v_out, "v_out")):
        if t is not None and t.shape != shape:
            raise ValueError(f"{what} has shape {tuple(t.shape)}, not {shape}")
    status = _calls.es_cache_read(cache.handle, batch.ref, _tensor(k_out, _BF16, "k_out"),
                                  _tensor(v_out, _BF16, "v_out"), _stream(stream))
    if status:
        _check(status, "es_cache_read")


def es_attention_workspace(cache: Cache, q_heads: int) -> int:
    """Bytes of (zeroed) workspace for es_attention with this cache, whatever the batch."""
    return int(_lib().es_attention_workspace(cache.handle, q_heads))


def es_attention_gave_up(workspace) -> bool:
    """Whether a kernel that used this workspace gave up a wait (an error of the library): its
    outputs since are not to be used, nor the workspace before it has been zeroed. Waits for the
    current stream; a program asks where it reads results anyway."""
    return bool(workspace[ES_ATTENTION_GAVE_UP:ES_ATTENTION_GAVE_UP + 4].any())


def es_attention(cache: Cache, batch: Batch, q, out, workspace, scale: float, lse=None,
                 softcap: float = 0.0, slopes=None, window: int = 0, first=None, last=None,
                 stream=None) -> None:
    """Attention of the batch's new tokens over the cache. ``q`` and ``out``: bfloat16
    [tokens, q_heads, head_dim]; ``lse``: float32 [tokens, q_heads]; ``workspace``: a zeroed
    uint8 tensor of es_attention_workspace() bytes, which every call leaves ready for the
    next on its stream."""
    d, n = cache.head_dim, batch.tokens
    q_ptr, q_stride, heads = _rows(q, n, None, d, "q")
    o_ptr, o_stride, _ = _rows(out, n, heads, d, "out")
    try:
        args = _ATTENTION.pack(
            q_ptr, o_ptr, _tensor(lse, _F32, "lse", n * heads), _tensor(slopes, _F32, "slopes", heads),
            _tensor(first, _I32, "first", n), _tensor(last, _I32, "last", n), q_stride, o_stride, heads,
            window, scale, softcap)
    except (_StructError, OverflowError) as e:
        raise ValueError(f"es_attention: {e}") from None
    status = _calls.es_attention(cache.handle, batch.ref, args, _tensor(workspace, _U8, "workspace"),
                                 workspace.numel(), _stream(stream))
    if status:
        _check(status, "es_attention")
