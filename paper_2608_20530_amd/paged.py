"""The paged cache of a serving program around the draft path: places for a step's tokens, head norms
with rotation into the cache, and the attentions that read it (include/lilicorr.h, "Paged cache").

Marshalling only, as in the rest of the package: torch supplies device memory and the current
stream, the library's kernels do the work. Single-token steps take a few microseconds on the GPU, so
the host's share counts: arguments are packed as bytes in the C structs' layout (a ctypes structure
filled by name takes 3 us), the stream is asked for as a number (2.8 us through a Stream object), and
checks read each property of a tensor once.
"""
from __future__ import annotations

import ctypes
import math
import struct
from typing import NamedTuple

import torch

from . import LilicorrError, lilicorr_status_string, load_library

__all__ = [
    "Cache", "PagePlanArgs", "QkNormRopeArgs", "AttentionArgs", "PagePlan", "lilicorr_page_plan",
    "lilicorr_qk_norm_rope", "lilicorr_window_attention", "lilicorr_prefix_attention",
    "lilicorr_window_attention_workspace_bytes", "lilicorr_prefix_attention_workspace_bytes",
    "page_plan", "qk_norm_rope", "window_attention", "window_attention_workspace",
    "prefix_attention", "prefix_attention_workspace",
]

P, I64, I, SZ, F = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float)
_CODE = {torch.bfloat16: 1, torch.float16: 2}
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32


class Cache(ctypes.Structure):
    """lilicorr_cache of include/lilicorr.h, field for field."""
    _fields_ = [("k", P), ("v", P), ("dtype", I), ("page_size", I), ("heads", I), ("d", I),
                ("pages", I64), ("page_stride", I64), ("token_stride", I64), ("head_stride", I64)]


class PagePlanArgs(ctypes.Structure):
    """lilicorr_page_plan_args of include/lilicorr.h, field for field."""
    _fields_ = [(n, P) for n in ("lengths", "incoming", "pages", "table", "queue", "cursor", "pages_out",
                                 "cursor_out", "starts", "totals", "slots", "positions")] + \
               [(n, I64) for n in ("N", "page_size", "table_width", "queue_size", "tokens", "window",
                                   "sinks")]


class QkNormRopeArgs(ctypes.Structure):
    """lilicorr_qk_norm_rope_args of include/lilicorr.h, field for field."""
    _fields_ = [("q", P), ("k", P), ("v", P), ("q_out", P), ("cache", Cache), ("slots", P),
                ("positions", P), ("cos_sin", P), ("q_weight", P), ("k_weight", P), ("q_stride", I64),
                ("k_stride", I64), ("v_stride", I64), ("tokens", I64), ("max_positions", I64),
                ("heads", I), ("rot", I), ("interleaved", I), ("eps", F)]


class AttentionArgs(ctypes.Structure):
    """lilicorr_attention_args of include/lilicorr.h, field for field."""
    _fields_ = [("q", P), ("out", P), ("cache", Cache), ("table", P), ("starts", P), ("totals", P),
                ("shared_table", P), ("workspace", P), ("workspace_bytes", SZ), ("tokens", I64),
                ("q_stride", I64), ("N", I64), ("table_width", I64), ("shared_length", I64),
                ("window", I64), ("sinks", I64), ("max_tokens", I64), ("max_length", I64),
                ("heads", I), ("causal", I), ("scale", F)]


# Each of these is the one that lilicorr_* of the same name takes: a Structure above, by reference, or
# its packed bytes.
SIGNATURES = {
    "lilicorr_page_plan": ([P, P], I),
    "lilicorr_qk_norm_rope": ([P, P], I),
    "lilicorr_window_attention": ([P, P], I),
    "lilicorr_prefix_attention": ([P, P], I),
    "lilicorr_window_attention_workspace_bytes": ([P], SZ),
    "lilicorr_prefix_attention_workspace_bytes": ([P], SZ),
}


def _packer(structure) -> struct.Struct:
    """A native-layout packer of the structure's fields in their order, nested ones in place."""
    letters = {P: "P", I64: "q", I: "i", SZ: "N", F: "f"}

    def of(s):
        return "".join(of(t) if issubclass(t, ctypes.Structure) else letters[t] for _, t in s._fields_)

    # the native alignment ends a struct at a multiple of its largest member, a pointer here
    return struct.Struct("@" + of(structure) + "0P")


_PLAN, _ROPE, _ATTENTION = _packer(PagePlanArgs), _packer(QkNormRopeArgs), _packer(AttentionArgs)


# ---- raw C ABI (same names as include/lilicorr.h) ------------------------------------------------

def _raw(name, args, stream) -> int:
    rc = getattr(load_library(), name)(args if isinstance(args, bytes) else ctypes.byref(args), stream)
    if rc != 0:
        raise LilicorrError(f"{name}: {lilicorr_status_string(rc)} (status {rc})")
    return rc


def lilicorr_page_plan(args: PagePlanArgs, stream) -> int:
    return _raw("lilicorr_page_plan", args, stream)


def lilicorr_qk_norm_rope(args: QkNormRopeArgs, stream) -> int:
    return _raw("lilicorr_qk_norm_rope", args, stream)


def lilicorr_window_attention(args: AttentionArgs, stream) -> int:
    return _raw("lilicorr_window_attention", args, stream)


def lilicorr_prefix_attention(args: AttentionArgs, stream) -> int:
    return _raw("lilicorr_prefix_attention", args, stream)


def lilicorr_window_attention_workspace_bytes(args: AttentionArgs) -> int:
    return load_library().lilicorr_window_attention_workspace_bytes(ctypes.byref(args))


def lilicorr_prefix_attention_workspace_bytes(args: AttentionArgs) -> int:
    return load_library().lilicorr_prefix_attention_workspace_bytes(ctypes.byref(args))


# ---- torch conveniences ------------------------------------------------------------------------

def _stream(t: torch.Tensor) -> int:
    """The current stream of the tensor's device, as a handle."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _ints(t: torch.Tensor, name: str, shape: tuple, dtype=_I32) -> int:
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
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
    the new tokens of the step). Where cursor[2] of the result is not 0 the queue ran out: request n has
    stored min(totals[n], pages[n, 0] * page_size) tokens, and the next step goes on from there. `out` must not share memory with the other arguments."""
    (N,), M, (C,) = lengths.shape, table.shape[-1], queue.shape
    n = (N,)
    if out is None:
        # one allocation, cut up: the cursor's 64-bit values first
        buf = torch.empty(7 + 4 * N + 2 * tokens, dtype=_I32, device=lengths.device)
        cur, pg, totals, starts, slots, positions = buf.split_with_sizes((6, 2 * N, N, N + 1, tokens, tokens))
        out = PagePlan(pg.view(N, 2), cur.view(_I64), starts, totals, slots, positions)
        at = buf.data_ptr()
        made = (at + 24, at, at + 24 + 12 * N, at + 24 + 8 * N, at + 28 + 16 * N,
                at + 28 + 16 * N + 4 * tokens)
    else:
        made = (_ints(out.pages, "out.pages", (N, 2)), _ints(out.cursor, "out.cursor", (3,), _I64),
                _ints(out.starts, "out.starts", (N + 1,)), _ints(out.totals, "out.totals", n),
                _ints(out.slots, "out.slots", (tokens,)),
                _ints(out.positions, "out.positions", (tokens,)))
    _raw("lilicorr_page_plan", _PLAN.pack(
        _ints(lengths, "lengths", n), _ints(incoming, "incoming", n), _ints(pages, "pages", (N, 2)),
        _ints(table, "table", (N, M)), _ints(queue, "queue", (C,)),
        _ints(cursor, "cursor", (3,), _I64), *made, N, page_size, M, C, tokens, window, sinks),
        _stream(lengths))
    return out


def _cache(k: torch.Tensor, v: torch.Tensor | None) -> tuple:
    """The fields of Cache for [pages, page_size, heads, d] views whose d elements lie in a row."""
    code, shape, strides = _CODE.get(k.dtype), k.shape, k.stride()
    if code is None or len(shape) != 4 or strides[3] != 1 or not k.is_cuda:
        raise LilicorrError("the cache must be bf16 or fp16 device tensors [pages, page_size, heads, d] "
                            f"with contiguous rows of d, got {k.dtype} {list(shape)} on {k.device}")
    if v is not None and (v.dtype is not k.dtype or v.shape != shape or v.stride() != strides or
                          not v.is_cuda):
        raise LilicorrError("k_cache and v_cache must have the same type, shape and strides")
    pages, size, heads, d = shape
    page, token, head, _ = strides  # of a dimension of one element torch's stride says nothing
    return (k.data_ptr(), 0 if v is None else v.data_ptr(), code, size, heads, d, pages,
            page if pages > 1 else 0, token if size > 1 else 0, head if heads > 1 else 0)


def _rows(t: torch.Tensor, name: str, shape: tuple, dtype) -> int:
    """Checks [tokens, heads, d] with whole heads side by side; -> elements from token to token."""
    step, head, one = t.stride() if t.dim() == 3 else (0, 0, 0)
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda:
        raise LilicorrError(f"{name} must be a {dtype} device tensor {list(shape)}, got "
                            f"{t.dtype} {list(t.shape)} on {t.device}")
    if one != 1 or (head != shape[2] and shape[1] > 1):
        raise LilicorrError(f"{name}: the heads of a token must lie side by side")
    return step if shape[0] > 1 else shape[1] * shape[2]


def _floats(t: torch.Tensor | None, name: str, shape: tuple) -> int:
    if t is None:
        return 0
    if t.dtype is not _F32 or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise LilicorrError(f"{name} must be a contiguous fp32 device tensor {list(shape)}, got "
                            f"{t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _output(out, like: torch.Tensor, shape: tuple, dtype) -> torch.Tensor:
    if out is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    if _rows(out, "out", shape, dtype) != shape[1] * shape[2]:
        raise LilicorrError("out must be contiguous")
    return out


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                 positions: torch.Tensor, cos_sin: torch.Tensor | None, k_cache: torch.Tensor,
                 v_cache: torch.Tensor, *, q_weight=None, k_weight=None, eps: float = 1e-6,
                 interleaved: bool = False, out=None) -> torch.Tensor:
    """q [T, heads, d], k and v [T, cache heads, d] (views of one projection's output will do): norms
    (where weights are given), rotation by cos_sin [positions, rot] fp32 (rot / 2 cosines, then as
    many sines), k and v into the caches at `slots` -> q [T, heads, d]."""
    cache, dtype = _cache(k_cache, v_cache), k_cache.dtype
    kv, d = cache[4], cache[5]
    shape = q.shape
    T, heads, _ = shape
    if shape[2] != d:
        raise LilicorrError(f"q has heads of {shape[2]}, the cache of {d}")
    most, rot = cos_sin.shape if cos_sin is not None else (0, 0)
    out = _output(out, q, shape, dtype)
    _raw("lilicorr_qk_norm_rope", _ROPE.pack(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), *cache, _ints(slots, "slots", (T,)),
        _ints(positions, "positions", (T,)), _floats(cos_sin, "cos_sin", (most, rot)),
        _floats(q_weight, "q_weight", (d,)), _floats(k_weight, "k_weight", (d,)),
        _rows(q, "q", shape, dtype), _rows(k, "k", (T, kv, d), dtype), _rows(v, "v", (T, kv, d), dtype),
        T, most, heads, rot, interleaved, eps), _stream(q))
    return out


def _pack_attention(q, out, k_cache, v_cache, pointers, workspace, table, shared_length, window, sinks,
                    causal, scale, max_tokens, max_length) -> bytes:
    cache = _cache(k_cache, v_cache)
    shape = q.shape
    T, heads, d = shape
    if d != cache[5]:
        raise LilicorrError(f"q has heads of {d}, the cache of {cache[5]}")
    N, M = table.shape
    return _ATTENTION.pack(
        q.data_ptr(), out, *cache, *pointers, *workspace, T, _rows(q, "q", shape, k_cache.dtype), N, M,
        shared_length, window, sinks, T if max_tokens is None else max_tokens,
        M * cache[3] if max_length is None else max_length, heads, causal,
        1 / math.sqrt(d) if scale is None else scale)


def _workspace(name, q, k_cache, table, shared_length, window, sinks, causal, max_tokens, max_length):
    need = getattr(load_library(), name + "_workspace_bytes")(_pack_attention(
        q, 0, k_cache, None, (0, 0, 0, 0), (0, 0), table, shared_length, window, sinks, causal, None,
        max_tokens, max_length))
    if need == 0:
        raise LilicorrError(f"{name} does not support these sizes")
    return torch.empty(need, dtype=torch.uint8, device=q.device)


def _attend(name, q, k_cache, v_cache, shared_table, shared_length, table, starts, totals, window, sinks,
            causal, scale, max_tokens, max_length, out, workspace) -> torch.Tensor:
    N, M = table.shape
    out = _output(out, q, q.shape, q.dtype)
    if workspace is None:
        workspace = _workspace(name, q, k_cache, table, shared_length, window, sinks, causal, max_tokens,
                               max_length)
    elif not workspace.is_cuda or not workspace.is_contiguous():
        raise LilicorrError("workspace must be a contiguous device tensor")
    pointers = (_ints(table, "table", (N, M)), _ints(starts, "starts", (N + 1,)),
                _ints(totals, "totals", (N,)), shared_table)
    _raw(name, _pack_attention(
        q, out.data_ptr(), k_cache, v_cache, pointers,
        (workspace.data_ptr(), workspace.numel() * workspace.element_size()), table, shared_length,
        window, sinks, causal, scale, max_tokens, max_length), _stream(q))
    return out


def window_attention_workspace(q: torch.Tensor, k_cache: torch.Tensor, table: torch.Tensor, *,
                               window: int = 0, sinks: int = 0, causal: bool = True,
                               max_tokens: int | None = None,
                               max_length: int | None = None) -> torch.Tensor:
    """A workspace for window_attention calls of these sizes, whose content does not matter."""
    return _workspace("lilicorr_window_attention", q, k_cache, table, 0, window, sinks, causal,
                      max_tokens, max_length)


def window_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     table: torch.Tensor, starts: torch.Tensor, totals: torch.Tensor, *,
                     window: int = 0, sinks: int = 0, causal: bool = True,
                     scale: float | None = None, max_tokens: int | None = None,
                     max_length: int | None = None, out=None, workspace=None) -> torch.Tensor:
    """q [T, heads, d] against caches [pages, page_size, cache heads, d] through table [N, M], with
    starts [N + 1] and totals [N] as page_plan makes them -> [T, heads, d]. window 0 is none; the
    scale is 1 / sqrt(d) unless given; max_tokens and max_length are upper bounds of a request's
    queries and keys that the host knows (all of q, the table's width unless given)."""
    return _attend("lilicorr_window_attention", q, k_cache, v_cache, 0, 0, table, starts, totals, window,
                   sinks, causal, scale, max_tokens, max_length, out, workspace)


def prefix_attention_workspace(q: torch.Tensor, k_cache: torch.Tensor, table: torch.Tensor,
                               shared_length: int, *, causal: bool = True,
                               max_tokens: int | None = None,
                               max_length: int | None = None) -> torch.Tensor:
    """A workspace for prefix_attention calls of these sizes, whose content does not matter."""
    return _workspace("lilicorr_prefix_attention", q, k_cache, table, shared_length, 0, 0, causal,
                      max_tokens, max_length)


def prefix_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     shared_table: torch.Tensor, shared_length: int, table: torch.Tensor,
                     starts: torch.Tensor, totals: torch.Tensor, *, causal: bool = True,
                     scale: float | None = None, max_tokens: int | None = None,
                     max_length: int | None = None, out=None, workspace=None) -> torch.Tensor:
    """window_attention without a window, for requests that all begin with the same shared_length
    tokens, whose pages shared_table lists; table, totals and positions count from their end on."""
    shared = _ints(shared_table, "shared_table", (-(-shared_length // k_cache.shape[1]),))
    return _attend("lilicorr_prefix_attention", q, k_cache, v_cache, shared, shared_length, table, starts,
                   totals, 0, 0, causal, scale, max_tokens, max_length, out, workspace)
