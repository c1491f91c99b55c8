"""The paged cache of a serving program around the draft path: places for a step's tokens, head norms
with rotation into the cache, and the attentions that read it (include/lilicorr.h, "Paged cache").

Marshalling only, as in the rest of the package: torch supplies device memory and the current
stream, the library's kernels do the work.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple

import torch

from . import LilicorrError, _call, _stream, load_library

__all__ = [
    "Cache", "AttentionArgs", "PagePlan", "lilicorr_page_plan", "lilicorr_qk_norm_rope",
    "lilicorr_window_attention", "lilicorr_prefix_attention",
    "lilicorr_window_attention_workspace_bytes", "lilicorr_prefix_attention_workspace_bytes",
    "page_plan", "qk_norm_rope", "window_attention", "window_attention_workspace",
    "prefix_attention", "prefix_attention_workspace",
]

P, I64, I, SZ, F = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float)
_CODE = {torch.bfloat16: 1, torch.float16: 2}


class Cache(ctypes.Structure):
    """lilicorr_cache of include/lilicorr.h, field for field."""
    _fields_ = [("k", P), ("v", P), ("dtype", I), ("page_size", I), ("heads", I), ("d", I),
                ("pages", I64), ("page_stride", I64), ("token_stride", I64), ("head_stride", I64)]


class AttentionArgs(ctypes.Structure):
    """lilicorr_attention_args of include/lilicorr.h, field for field."""
    _fields_ = [("q", P), ("out", P), ("cache", Cache), ("table", P), ("starts", P), ("totals", P),
                ("shared_table", P), ("workspace", P), ("workspace_bytes", SZ), ("tokens", I64),
                ("q_stride", I64), ("N", I64), ("table_width", I64), ("shared_length", I64),
                ("window", I64), ("sinks", I64), ("max_tokens", I64), ("max_length", I64),
                ("heads", I), ("causal", I), ("scale", F)]


SIGNATURES = {
    "lilicorr_page_plan": ([P] * 6 + [I64, I] + [I64] * 5 + [P] * 7, I),
    "lilicorr_qk_norm_rope": ([P, I64, I, P, I64, P, I64, I64, P, P, P, I64, I, I, P, P, F,
                               ctypes.POINTER(Cache), P, P], I),
    "lilicorr_window_attention": ([ctypes.POINTER(AttentionArgs), P], I),
    "lilicorr_prefix_attention": ([ctypes.POINTER(AttentionArgs), P], I),
    "lilicorr_window_attention_workspace_bytes": ([ctypes.POINTER(AttentionArgs)], SZ),
    "lilicorr_prefix_attention_workspace_bytes": ([ctypes.POINTER(AttentionArgs)], SZ),
}


# ---- raw C ABI (same names and argument order as include/lilicorr.h) ----------------------------

def lilicorr_page_plan(lengths, incoming, pages, table, queue, cursor, N, page_size, table_width,
                       queue_size, tokens, window, sinks, pages_out, cursor_out, starts, totals,
                       slots, positions, stream):
    return _call("lilicorr_page_plan", lengths, incoming, pages, table, queue, cursor, N, page_size,
                 table_width, queue_size, tokens, window, sinks, pages_out, cursor_out, starts,
                 totals, slots, positions, stream)


def lilicorr_qk_norm_rope(q, q_stride, heads, k, k_stride, v, v_stride, tokens, slots, positions,
                          cos_sin, max_positions, rot, interleaved, q_weight, k_weight, eps,
                          cache: Cache, q_out, stream):
    return _call("lilicorr_qk_norm_rope", q, q_stride, heads, k, k_stride, v, v_stride, tokens,
                 slots, positions, cos_sin, max_positions, rot, interleaved, q_weight, k_weight,
                 eps, cache, q_out, stream)


def lilicorr_window_attention(args: AttentionArgs, stream):
    return _call("lilicorr_window_attention", args, stream)


def lilicorr_prefix_attention(args: AttentionArgs, stream):
    return _call("lilicorr_prefix_attention", args, stream)


def lilicorr_window_attention_workspace_bytes(args: AttentionArgs) -> int:
    return load_library().lilicorr_window_attention_workspace_bytes(args)


def lilicorr_prefix_attention_workspace_bytes(args: AttentionArgs) -> int:
    return load_library().lilicorr_prefix_attention_workspace_bytes(args)


# ---- torch conveniences ------------------------------------------------------------------------

def _ints(t: torch.Tensor, name: str, shape, dtype=torch.int32) -> int:
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != shape:
        raise LilicorrError(f"{name} must be a contiguous {dtype} device tensor {list(shape)}, got "
                            f"{t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


class PagePlan(NamedTuple):
    """What page_plan makes. pages and cursor go into the next step's call."""
    pages: torch.Tensor      # [N, 2] int32
    cursor: torch.Tensor     # [3] int64: head, tail, pages that were lacking
    starts: torch.Tensor     # [N + 1] int32
    totals: torch.Tensor     # [N] int32
    slots: torch.Tensor      # [tokens] int32
    positions: torch.Tensor  # [tokens] int32


def page_plan(lengths: torch.Tensor, incoming: torch.Tensor, pages: torch.Tensor,
              table: torch.Tensor, queue: torch.Tensor, cursor: torch.Tensor, *, page_size: int,
              tokens: int, window: int = 0, sinks: int = 0, out: PagePlan | None = None) -> PagePlan:
    """One step's places. lengths, incoming [N], pages [N, 2] int32; table [N, M] and queue [C] int32
    are updated in place; cursor [3] int64. `tokens` rows of slots and positions are made (at least
    the new tokens of the step). `out` must not share memory with `pages` or `cursor`."""
    N, M, C = lengths.shape[0], table.shape[1], queue.shape[0]
    if out is None:
        # one allocation, cut up: cursor first (8-byte elements)
        buf = torch.empty(6 + 4 * N + 1 + 2 * tokens, dtype=torch.int32, device=lengths.device)
        cur, pg, st, tot, sl, ps = buf.split((6, 2 * N, N + 1, N, tokens, tokens))
        out = PagePlan(pg.view(N, 2), cur.view(torch.int64), st, tot, sl, ps)
    lilicorr_page_plan(_ints(lengths, "lengths", (N,)), _ints(incoming, "incoming", (N,)),
                       _ints(pages, "pages", (N, 2)), _ints(table, "table", (N, M)),
                       _ints(queue, "queue", (C,)), _ints(cursor, "cursor", (3,), torch.int64), N,
                       page_size, M, C, tokens, window, sinks, _ints(out.pages, "out.pages", (N, 2)),
                       _ints(out.cursor, "out.cursor", (3,), torch.int64),
                       _ints(out.starts, "out.starts", (N + 1,)),
                       _ints(out.totals, "out.totals", (N,)),
                       _ints(out.slots, "out.slots", (tokens,)),
                       _ints(out.positions, "out.positions", (tokens,)), _stream())
    return out


def _cache(k_cache: torch.Tensor, v_cache: torch.Tensor | None) -> Cache:
    """[pages, page_size, heads, d] views of any strides that end in d elements in a row."""
    if k_cache.dtype not in _CODE or not k_cache.is_cuda or k_cache.dim() != 4:
        raise LilicorrError("the cache must be bf16 or fp16 device tensors [pages, page_size, heads, d]")
    page, token, head, one = k_cache.stride()
    if one != 1:
        raise LilicorrError("the cache's innermost dimension must be contiguous")
    if v_cache is not None and (v_cache.dtype != k_cache.dtype or v_cache.shape != k_cache.shape or
                                v_cache.stride() != k_cache.stride() or not v_cache.is_cuda):
        raise LilicorrError("k_cache and v_cache must have the same type, shape and strides")
    pages, size, heads, d = k_cache.shape
    return Cache(k_cache.data_ptr(), v_cache.data_ptr() if v_cache is not None else None,
                 _CODE[k_cache.dtype], size, heads, d, pages, page, token, head)


def _rows(t: torch.Tensor, name: str, tokens: int, heads: int, d: int, dtype) -> int:
    """Checks [tokens, heads, d] with whole heads side by side; -> elements from token to token."""
    if t.dtype != dtype or not t.is_cuda or tuple(t.shape) != (tokens, heads, d):
        raise LilicorrError(f"{name} must be a {dtype} device tensor {[tokens, heads, d]}, got "
                            f"{t.dtype} {list(t.shape)} on {t.device}")
    step, head, one = t.stride()
    if one != 1 or (head != d and heads > 1):
        raise LilicorrError(f"{name}: the heads of a token must lie side by side")
    return step if tokens > 1 else heads * d


def _weights(t: torch.Tensor | None, name: str, d: int):
    if t is None:
        return None
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != (d,):
        raise LilicorrError(f"{name} must be a contiguous fp32 device tensor [{d}]")
    return t.data_ptr()


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                 positions: torch.Tensor, cos_sin: torch.Tensor | None, k_cache: torch.Tensor,
                 v_cache: torch.Tensor, *, q_weight=None, k_weight=None, eps: float = 1e-6,
                 interleaved: bool = False, out=None) -> torch.Tensor:
    """q [T, heads, d], k and v [T, cache heads, d] (views of one projection's output will do): norms
    (where weights are given), rotation by cos_sin [positions, rot] fp32 (rot / 2 cosines, then as
    many sines), k and v into the caches at `slots` -> q [T, heads, d]."""
    c = _cache(k_cache, v_cache)
    T, heads, d = q.shape
    kv, dtype = c.heads, k_cache.dtype
    if d != c.d:
        raise LilicorrError(f"q has heads of {d}, the cache of {c.d}")
    strides = (_rows(q, "q", T, heads, d, dtype), _rows(k, "k", T, kv, d, dtype),
               _rows(v, "v", T, kv, d, dtype))
    most = rot = 0
    if cos_sin is not None:
        most, rot = cos_sin.shape
        if cos_sin.dtype != torch.float32 or not cos_sin.is_cuda or not cos_sin.is_contiguous():
            raise LilicorrError("cos_sin must be a contiguous fp32 device tensor [positions, rot]")
    if out is None:
        out = torch.empty(T, heads, d, dtype=dtype, device=q.device)
    elif _rows(out, "out", T, heads, d, dtype) != heads * d:
        raise LilicorrError("out must be contiguous")
    lilicorr_qk_norm_rope(q.data_ptr(), strides[0], heads, k.data_ptr(), strides[1], v.data_ptr(),
                          strides[2], T, _ints(slots, "slots", (T,)),
                          _ints(positions, "positions", (T,)),
                          cos_sin.data_ptr() if cos_sin is not None else None, most, rot,
                          int(interleaved), _weights(q_weight, "q_weight", d),
                          _weights(k_weight, "k_weight", d), eps, c, out.data_ptr(), _stream())
    return out


def _attention_args(q, k_cache, v_cache, table, window, sinks, causal, scale, max_tokens, max_length,
                    shared_length) -> AttentionArgs:
    c = _cache(k_cache, v_cache)
    T, heads, d = q.shape
    if d != c.d:
        raise LilicorrError(f"q has heads of {d}, the cache of {c.d}")
    N, M = table.shape
    return AttentionArgs(
        q=q.data_ptr(), cache=c, tokens=T, q_stride=_rows(q, "q", T, heads, d, k_cache.dtype), N=N,
        table_width=M, shared_length=shared_length, window=window, sinks=sinks,
        max_tokens=T if max_tokens is None else max_tokens,
        max_length=M * c.page_size if max_length is None else max_length, heads=heads,
        causal=int(causal), scale=1 / math.sqrt(d) if scale is None else scale)


def _attend(name, a: AttentionArgs, q, table, starts, totals, out, workspace):
    N, M = table.shape
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif _rows(out, "out", *q.shape, q.dtype) != q.shape[1] * q.shape[2]:
        raise LilicorrError("out must be contiguous")
    if workspace is None:
        workspace = _workspace(name, a, q.device)
    elif not workspace.is_cuda or not workspace.is_contiguous():
        raise LilicorrError("workspace must be a contiguous device tensor")
    a.out, a.table = out.data_ptr(), _ints(table, "table", (N, M))
    a.starts, a.totals = _ints(starts, "starts", (N + 1,)), _ints(totals, "totals", (N,))
    a.workspace = workspace.data_ptr()
    a.workspace_bytes = workspace.numel() * workspace.element_size()
    _call(name, a, _stream())
    return out


def _workspace(name, a: AttentionArgs, device) -> torch.Tensor:
    need = getattr(load_library(), name + "_workspace_bytes")(a)
    if need == 0:
        raise LilicorrError(f"{name} does not support these sizes")
    return torch.zeros(need, dtype=torch.uint8, device=device)


def window_attention_workspace(q: torch.Tensor, k_cache: torch.Tensor, table: torch.Tensor, *,
                               window: int = 0, sinks: int = 0, causal: bool = True,
                               max_tokens: int | None = None,
                               max_length: int | None = None) -> torch.Tensor:
    """A zero-filled workspace for window_attention calls of these sizes (kept ready by the calls)."""
    a = _attention_args(q, k_cache, None, table, window, sinks, causal, None, max_tokens, max_length, 0)
    return _workspace("lilicorr_window_attention", a, q.device)


def window_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     table: torch.Tensor, starts: torch.Tensor, totals: torch.Tensor, *,
                     window: int = 0, sinks: int = 0, causal: bool = True,
                     scale: float | None = None, max_tokens: int | None = None,
                     max_length: int | None = None, out=None, workspace=None) -> torch.Tensor:
    """q [T, heads, d] against caches [pages, page_size, cache heads, d] through table [N, M], with
    starts [N + 1] and totals [N] as page_plan makes them -> [T, heads, d]. window 0 is none; the
    scale is 1 / sqrt(d) unless given; max_tokens and max_length are upper bounds of a request's
    queries and keys that the host knows (all of q, the table's width unless given)."""
    a = _attention_args(q, k_cache, v_cache, table, window, sinks, causal, scale, max_tokens,
                        max_length, 0)
    return _attend("lilicorr_window_attention", a, q, table, starts, totals, out, workspace)


def prefix_attention_workspace(q: torch.Tensor, k_cache: torch.Tensor, table: torch.Tensor,
                               shared_length: int, *, causal: bool = True,
                               max_tokens: int | None = None,
                               max_length: int | None = None) -> torch.Tensor:
    """A zero-filled workspace for prefix_attention calls of these sizes (kept ready by the calls)."""
    a = _attention_args(q, k_cache, None, table, 0, 0, causal, None, max_tokens, max_length,
                        shared_length)
    return _workspace("lilicorr_prefix_attention", a, q.device)


def prefix_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     shared_table: torch.Tensor, shared_length: int, table: torch.Tensor,
                     starts: torch.Tensor, totals: torch.Tensor, *, causal: bool = True,
                     scale: float | None = None, max_tokens: int | None = None,
                     max_length: int | None = None, out=None, workspace=None) -> torch.Tensor:
    """window_attention without a window, for requests that all begin with the same shared_length
    tokens, whose pages shared_table lists; table, totals and positions count from their end on."""
    a = _attention_args(q, k_cache, v_cache, table, 0, 0, causal, scale, max_tokens, max_length,
                        shared_length)
    a.shared_table = _ints(shared_table, "shared_table",
                           (-(-shared_length // k_cache.shape[1]),))
    return _attend("lilicorr_prefix_attention", a, q, table, starts, totals, out, workspace)
