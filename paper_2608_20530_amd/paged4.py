"""The paged cache in 4 bits: its writer, the attention that reads it, the attention weight that its keys have got,
and eviction by that weight (include/lilicorr.h, "The cache in 4 bits"). Places, tables, starts and totals are
page_plan's.

Marshalling only, in the manner of paged.py: arguments are packed as bytes in the C structs' layout.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple

import torch

from . import LilicorrError, load_library
from .paged import _CODE, _F32, _I64, F, I, I64, P, SZ, _floats, _ints, _output, _packer, _raw, _rows, _stream

__all__ = [
    "Cache4Args", "QkNormRope4Args", "Attention4Args", "KeyWeightsArgs", "EvictArgs", "Cache4", "Eviction",
    "lilicorr_qk_norm_rope4", "lilicorr_window_attention4", "lilicorr_window_attention4_workspace_bytes",
    "lilicorr_key_weights", "lilicorr_evict", "lilicorr_evict_workspace_bytes",
    "cache4", "qk_norm_rope4", "window_attention4", "window_attention4_workspace", "key_weights", "evict",
    "evict_workspace",
]

_U8 = torch.uint8


class Cache4Args(ctypes.Structure):
    """lilicorr_cache4 of include/lilicorr.h, field for field."""
    _fields_ = [("k", P), ("v", P), ("k_scales", P), ("v_scales", P), ("page_size", I), ("heads", I), ("d", I),
                ("pages", I64), ("page_stride", I64), ("token_stride", I64), ("head_stride", I64)]


class QkNormRope4Args(ctypes.Structure):
    """lilicorr_qk_norm_rope4_args of include/lilicorr.h, field for field."""
    _fields_ = [("q", P), ("k", P), ("v", P), ("q_out", P), ("cache", Cache4Args), ("slots", P), ("positions", P),
                ("cos_sin", P), ("q_weight", P), ("k_weight", P), ("q_stride", I64), ("k_stride", I64),
                ("v_stride", I64), ("tokens", I64), ("max_positions", I64), ("dtype", I), ("heads", I), ("rot", I),
                ("interleaved", I), ("eps", F)]


class Attention4Args(ctypes.Structure):
    """lilicorr_attention4_args of include/lilicorr.h, field for field."""
    _fields_ = [("q", P), ("out", P), ("lse", P), ("cache", Cache4Args), ("table", P), ("starts", P), ("totals", P),
                ("workspace", P), ("workspace_bytes", SZ), ("tokens", I64), ("q_stride", I64), ("N", I64),
                ("table_width", I64), ("window", I64), ("sinks", I64), ("max_tokens", I64), ("max_length", I64),
                ("dtype", I), ("heads", I), ("causal", I), ("scale", F)]


class KeyWeightsArgs(ctypes.Structure):
    """lilicorr_key_weights_args of include/lilicorr.h, field for field."""
    _fields_ = [("q", P), ("lse", P), ("weights", P), ("cache", Cache4Args), ("table", P), ("starts", P),
                ("totals", P), ("tokens", I64), ("q_stride", I64), ("N", I64), ("table_width", I64),
                ("max_tokens", I64), ("max_length", I64), ("dtype", I), ("heads", I), ("causal", I), ("scale", F),
                ("decay", F)]


class EvictArgs(ctypes.Structure):
    """lilicorr_evict_args of include/lilicorr.h, field for field."""
    _fields_ = [("cache", Cache4Args)] + \
               [(n, P) for n in ("weights", "table", "totals", "pages", "queue", "cursor", "totals_out", "pages_out",
                                 "evicted", "cursor_out", "workspace")] + [("workspace_bytes", SZ)] + \
               [(n, I64) for n in ("N", "table_width", "queue_size", "max_length", "budget", "limit", "sinks",
                                   "recent")]


SIGNATURES = {
    "lilicorr_qk_norm_rope4": ([P, P], I),
    "lilicorr_window_attention4": ([P, P], I),
    "lilicorr_window_attention4_workspace_bytes": ([P], SZ),
    "lilicorr_key_weights": ([P, P], I),
    "lilicorr_evict": ([P, P], I),
    "lilicorr_evict_workspace_bytes": ([P], SZ),
}

_ROPE, _ATTENTION, _WEIGHTS, _EVICT = map(_packer, (QkNormRope4Args, Attention4Args, KeyWeightsArgs, EvictArgs))


# ---- raw C ABI (same names as include/lilicorr.h) ------------------------------------------------

def lilicorr_qk_norm_rope4(args: QkNormRope4Args, stream) -> int:
    return _raw("lilicorr_qk_norm_rope4", args, stream)


def lilicorr_window_attention4(args: Attention4Args, stream) -> int:
    return _raw("lilicorr_window_attention4", args, stream)


def lilicorr_key_weights(args: KeyWeightsArgs, stream) -> int:
    return _raw("lilicorr_key_weights", args, stream)


def lilicorr_evict(args: EvictArgs, stream) -> int:
    return _raw("lilicorr_evict", args, stream)


def lilicorr_window_attention4_workspace_bytes(args: Attention4Args) -> int:
    return load_library().lilicorr_window_attention4_workspace_bytes(ctypes.byref(args))


def lilicorr_evict_workspace_bytes(args: EvictArgs) -> int:
    return load_library().lilicorr_evict_workspace_bytes(ctypes.byref(args))


# ---- torch conveniences ------------------------------------------------------------------------

class Cache4(NamedTuple):
    """Codes [pages, page_size, heads, d / 2] and scales [pages, page_size, heads, d / 32], uint8, of keys and
    values (None where a call reads keys alone). Any strides that are multiples of 16 bytes (codes; a row of codes lies
    together), scales laid out as codes are, at a sixteenth of the distances."""
    k: torch.Tensor
    k_scales: torch.Tensor
    v: torch.Tensor | None
    v_scales: torch.Tensor | None


def cache4(pages: int, page_size: int, heads: int, d: int, device="cuda") -> Cache4:
    """An empty cache: every element 0."""
    codes = lambda: torch.zeros(pages, page_size, heads, d // 2, dtype=_U8, device=device)  # noqa: E731
    scales = lambda: torch.ones(pages, page_size, heads, d // 32, dtype=_U8, device=device)  # noqa: E731
    if d % 32:
        raise LilicorrError(f"heads of {d}: a 4-bit cache has blocks of 32 elements")
    return Cache4(codes(), scales(), codes(), scales())


def _part(codes, scales, name: str, shape: tuple, strides: tuple) -> tuple:
    """Checks one of keys and values against the keys' shape and strides; -> the two addresses."""
    if (codes.dtype is not _U8 or scales.dtype is not _U8 or codes.dim() != 4 or not codes.is_cuda or
            not scales.is_cuda or codes.stride(3) != 1):
        raise LilicorrError(f"the cache's {name} must be uint8 device tensors [pages, page_size, heads, d / 2] with "
                            f"contiguous rows and [pages, page_size, heads, d / 32], got {codes.dtype} "
                            f"{list(codes.shape)} on {codes.device} and {scales.dtype} {list(scales.shape)} on "
                            f"{scales.device}")
    if codes.shape != shape or scales.shape != (*shape[:3], shape[3] // 16) or shape[3] % 16:
        raise LilicorrError(f"the cache's {name} must have codes {list(shape)}, with a multiple of 16 bytes a head, and "
                            f"scales [.., {shape[3] // 16}], got {list(codes.shape)} and {list(scales.shape)}")
    # of a dimension of one element torch's stride says nothing
    got, sc = codes.stride(), scales.stride()
    for i in range(3):
        if shape[i] > 1 and (got[i] != strides[i] or got[i] != 16 * sc[i]):
            raise LilicorrError(f"the cache's {name}: scales must be laid out as codes, at a sixteenth of their strides, "
                                f"and values as keys; got strides {got} and {sc}, keys {strides}")
    if shape[3] > 16 and sc[3] != 1:
        raise LilicorrError(f"the cache's {name}: the scales of a head must lie side by side")
    return codes.data_ptr(), scales.data_ptr()


def _cache(c: Cache4, values: bool = True) -> tuple:
    """The fields of Cache4Args."""
    if c.k is None or c.k_scales is None or (values and (c.v is None or c.v_scales is None)):
        raise LilicorrError(f"this call needs the cache's keys{' and values' if values else ''}, codes and scales")
    shape, strides = c.k.shape, c.k.stride()
    k, ks = _part(c.k, c.k_scales, "keys", shape, strides)
    v, vs = _part(c.v, c.v_scales, "values", shape, strides) if values else (0, 0)
    pages, size, heads, half = shape
    return (k, v, ks, vs, size, heads, 2 * half, pages, strides[0] if pages > 1 else 0,
            strides[1] if size > 1 else 0, strides[2] if heads > 1 else 0)


def _code(t: torch.Tensor, name: str) -> int:
    code = _CODE.get(t.dtype)
    if code is None:
        raise LilicorrError(f"{name} must be bf16 or fp16, got {t.dtype}")
    return code


def qk_norm_rope4(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: torch.Tensor,
                  cos_sin: torch.Tensor | None, cache: Cache4, *, q_weight=None, k_weight=None, eps: float = 1e-6,
                  interleaved: bool = False, out=None) -> torch.Tensor:
    """qk_norm_rope into a 4-bit cache: q [T, heads, d], k and v [T, cache heads, d] bf16 or fp16 (views of one
    projection's output will do), k and v in 4 bits into the cache at `slots` -> q [T, heads, d]."""
    c, dtype = _cache(cache), q.dtype
    code, kv, d = _code(q, "q"), c[5], c[6]
    shape = q.shape
    T, heads, _ = shape
    if shape[2] != d:
        raise LilicorrError(f"q has heads of {shape[2]}, the cache of {d}")
    most, rot = cos_sin.shape if cos_sin is not None else (0, 0)
    out = _output(out, q, shape, dtype)
    _raw("lilicorr_qk_norm_rope4", _ROPE.pack(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), *c, _ints(slots, "slots", (T,)),
        _ints(positions, "positions", (T,)), _floats(cos_sin, "cos_sin", (most, rot)),
        _floats(q_weight, "q_weight", (d,)), _floats(k_weight, "k_weight", (d,)),
        _rows(q, "q", shape, dtype), _rows(k, "k", (T, kv, d), dtype), _rows(v, "v", (T, kv, d), dtype),
        T, most, code, heads, rot, interleaved, eps), _stream(q))
    return out


def _pack_attention(q, out, lse, c, pointers, workspace, table, window, sinks, causal, scale, max_tokens,
                    max_length) -> bytes:
    shape = q.shape
    T, heads, d = shape
    if d != c[6]:
        raise LilicorrError(f"q has heads of {d}, the cache of {c[6]}")
    N, M = table.shape
    return _ATTENTION.pack(
        q.data_ptr(), out, lse, *c, *pointers, *workspace, T, _rows(q, "q", shape, q.dtype), N, M, window, sinks,
        T if max_tokens is None else max_tokens, M * c[4] if max_length is None else max_length, _code(q, "q"), heads,
        causal, 1 / math.sqrt(d) if scale is None else scale)


def window_attention4_workspace(q: torch.Tensor, cache: Cache4, table: torch.Tensor, *, window: int = 0, sinks: int = 0,
                                causal: bool = True, max_tokens: int | None = None,
                                max_length: int | None = None) -> torch.Tensor:
    """A workspace for window_attention4 calls of these sizes, whose content does not matter."""
    need = load_library().lilicorr_window_attention4_workspace_bytes(_pack_attention(
        q, 0, 0, _cache(cache), (0, 0, 0), (0, 0), table, window, sinks, causal, None, max_tokens, max_length))
    if need == 0:
        raise LilicorrError("lilicorr_window_attention4 does not support these sizes")
    return torch.empty(need, dtype=_U8, device=q.device)


def _space(workspace, make) -> tuple:
    """-> the workspace (which must live until the launch), its address and size."""
    if workspace is None:
        workspace = make()
    elif not workspace.is_cuda or not workspace.is_contiguous():
        raise LilicorrError("workspace must be a contiguous device tensor")
    return workspace, (workspace.data_ptr(), workspace.numel() * workspace.element_size())


def window_attention4(q: torch.Tensor, cache: Cache4, table: torch.Tensor, starts: torch.Tensor, totals: torch.Tensor, *,
                      window: int = 0, sinks: int = 0, causal: bool = True, scale: float | None = None,
                      max_tokens: int | None = None, max_length: int | None = None, lse=None, out=None,
                      workspace=None) -> torch.Tensor:
    """window_attention over a 4-bit cache: q [T, heads, d] bf16 or fp16 -> [T, heads, d]. `lse` [T, heads] fp32
    receives the logarithm of each row's sum of exponentials, for key_weights. The other arguments are
    window_attention's."""
    N, M = table.shape
    T, heads, _ = q.shape
    out = _output(out, q, q.shape, q.dtype)
    workspace, space = _space(workspace, lambda: window_attention4_workspace(
        q, cache, table, window=window, sinks=sinks, causal=causal, max_tokens=max_tokens, max_length=max_length))
    pointers = (_ints(table, "table", (N, M)), _ints(starts, "starts", (N + 1,)), _ints(totals, "totals", (N,)))
    _raw("lilicorr_window_attention4", _pack_attention(
        q, out.data_ptr(), _floats(lse, "lse", (T, heads)), _cache(cache), pointers, space, table, window, sinks,
        causal, scale, max_tokens, max_length), _stream(q))
    return out


def key_weights(q: torch.Tensor, lse: torch.Tensor, cache: Cache4, table: torch.Tensor, starts: torch.Tensor,
                totals: torch.Tensor, weights: torch.Tensor, *, causal: bool = True, scale: float | None = None,
                decay: float = 1.0, max_tokens: int | None = None, max_length: int | None = None) -> torch.Tensor:
    """Adds to `weights` [pages, cache heads, page_size] fp32 what attention the queries of this step gave to every key:
    q and the rest as window_attention4 had them, without a window, and the lse that it made. Weights of earlier steps
    count `decay` times; those of the step's own keys start anew. -> weights"""
    c = _cache(cache, False)
    shape = q.shape
    T, heads, d = shape
    if d != c[6]:
        raise LilicorrError(f"q has heads of {d}, the cache of {c[6]}")
    if lse is None:
        raise LilicorrError("key_weights needs the attention's lse")
    N, M = table.shape
    _raw("lilicorr_key_weights", _WEIGHTS.pack(
        q.data_ptr(), _floats(lse, "lse", (T, heads)), _floats(weights, "weights", (c[7], c[5], c[4])), *c,
        _ints(table, "table", (N, M)), _ints(starts, "starts", (N + 1,)), _ints(totals, "totals", (N,)), T,
        _rows(q, "q", shape, q.dtype), N, M, T if max_tokens is None else max_tokens,
        M * c[4] if max_length is None else max_length, _code(q, "q"), heads, causal,
        1 / math.sqrt(d) if scale is None else scale, decay), _stream(q))
    return weights


class Eviction(NamedTuple):
    """What evict makes. totals are the next step's lengths; pages and cursor go into its page_plan."""
    totals: torch.Tensor   # [N] int32
    pages: torch.Tensor    # [N, 2] int32
    cursor: torch.Tensor   # [3] int64
    evicted: torch.Tensor  # [N] int32: tokens that the request lost


def _pack_evict(c, pointers, workspace, N, M, C, max_length, budget, limit, sinks, recent) -> bytes:
    return _EVICT.pack(*c, *pointers, *workspace, N, M, C, M * c[4] if max_length is None else max_length, budget,
                       budget if limit is None else limit, sinks, recent)


def evict_workspace(cache: Cache4, table: torch.Tensor, *, budget: int, max_length: int | None = None) -> torch.Tensor:
    """A workspace for evict calls of these sizes, whose content does not matter."""
    N, M = table.shape
    need = load_library().lilicorr_evict_workspace_bytes(_pack_evict(
        _cache(cache), (0,) * 10, (0, 0), N, M, 1, max_length, budget, None, 0, 0))
    if need == 0:
        raise LilicorrError("lilicorr_evict does not support these sizes")
    return torch.empty(need, dtype=_U8, device=table.device)


def evict(cache: Cache4, weights: torch.Tensor, table: torch.Tensor, totals: torch.Tensor, pages: torch.Tensor,
          queue: torch.Tensor, cursor: torch.Tensor, *, budget: int, limit: int | None = None, sinks: int = 0,
          recent: int = 0, max_length: int | None = None, out: Eviction | None = None, workspace=None) -> Eviction:
    """Cuts every request of more than `limit` tokens (the budget unless given) to `budget`: each cache head keeps the
    first `sinks`, the last `recent` and the heaviest of the others by `weights`, moved to the front in their order.
    totals [N], pages [N, 2], cursor [3] are those of the step's page_plan (or of window-less ones before); table is
    read, the cache, weights and queue are updated in place. The next page_plan takes the result's totals as
    lengths; give its tokens the positions that it says plus all that `evicted` has said of their request."""
    N, M = table.shape
    n, C = (N,), queue.shape[0]
    if out is None:
        # one allocation, cut up: the cursor's 64-bit values first
        buf = torch.empty(6 + 4 * N, dtype=torch.int32, device=table.device)
        cur, pg, tot, lost = buf.split_with_sizes((6, 2 * N, N, N))
        out = Eviction(tot, pg.view(N, 2), cur.view(_I64), lost)
        at = buf.data_ptr()
        made = (at + 24 + 8 * N, at + 24, at + 24 + 12 * N, at)
    else:
        made = (_ints(out.totals, "out.totals", n), _ints(out.pages, "out.pages", (N, 2)),
                _ints(out.evicted, "out.evicted", n), _ints(out.cursor, "out.cursor", (3,), _I64))
    c = _cache(cache)
    workspace, space = _space(workspace, lambda: evict_workspace(cache, table, budget=budget, max_length=max_length))
    if weights.dtype is not _F32:
        raise LilicorrError(f"weights must be fp32, got {weights.dtype}")
    _raw("lilicorr_evict", _pack_evict(
        c, (_floats(weights, "weights", (c[7], c[5], c[4])), _ints(table, "table", (N, M)), _ints(totals, "totals", n),
            _ints(pages, "pages", (N, 2)), _ints(queue, "queue", (C,)), _ints(cursor, "cursor", (3,), _I64), *made),
        space, N, M, C, max_length, budget, limit, sinks, recent), _stream(table))
    return out
