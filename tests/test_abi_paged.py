"""Host-side checks of the paged-cache calls (no GPU): the packed bytes are the C structs' layout, and
bad arguments are refused before anything is launched."""
import ctypes

import pytest
import torch

import paper_2608_20530_amd as L
from paper_2608_20530_amd import paged

A = 4096  # a fake, 16-byte aligned "device" address: never dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    return L.load_library()


@pytest.mark.parametrize("packer,structure", [(paged._PLAN, L.PagePlanArgs), (paged._ROPE, L.QkNormRopeArgs),
                                              (paged._ATTENTION, L.AttentionArgs)])
def test_packed_bytes_are_the_struct(packer, structure):
    assert packer.size == ctypes.sizeof(structure)
    count = len(packer.unpack(bytes(packer.size)))
    raw = packer.pack(*range(1, count + 1))
    x = structure.from_buffer_copy(raw)
    flat = []
    for name, kind in structure._fields_:
        v = getattr(x, name)
        flat += [getattr(v, n) for n, _ in kind._fields_] if isinstance(v, ctypes.Structure) else [v]
    assert flat == list(range(1, count + 1))


def _plan(**changes):
    x = L.PagePlanArgs(**{n: A for n, t in L.PagePlanArgs._fields_ if t is ctypes.c_void_p},
                       N=4, page_size=16, table_width=8, queue_size=64, tokens=10, window=0, sinks=0)
    x.pages_out, x.cursor_out = 2 * A, 2 * A
    for k, v in changes.items():
        setattr(x, k, v)
    return x


@pytest.mark.parametrize("changes,status", [
    *[({n: None}, -1) for n in ("lengths", "incoming", "pages", "table", "queue", "cursor", "pages_out",
                                "cursor_out", "starts", "totals", "slots", "positions")],
    (dict(N=0), -1), (dict(page_size=0), -1), (dict(table_width=0), -1), (dict(queue_size=0), -1),
    (dict(tokens=-1), -1), (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(sinks=4), -1),
    (dict(pages_out=A), -1), (dict(cursor_out=A), -1),
    (dict(N=4097), -2), (dict(page_size=65537), -2), (dict(table_width=1 << 28), -2),
    (dict(queue_size=1 << 31), -2), (dict(tokens=1 << 31), -2), (dict(window=1 << 31), -2),
    (dict(lengths=A + 2), -3), (dict(cursor=A + 4), -3), (dict(slots=A + 1), -3),
])
def test_page_plan_refusals(lib, changes, status):
    assert lib.lilicorr_page_plan(ctypes.byref(_plan(**changes)), None) == status


def _cache(**changes):
    c = dict(k=A, v=A, dtype=1, page_size=16, heads=2, d=64, pages=10, page_stride=2048, token_stride=128,
             head_stride=64)
    return L.Cache(**dict(c, **changes))


CACHE_REFUSALS = [(dict(dtype=0), -1), (dict(dtype=3), -1), (dict(page_size=0), -1), (dict(heads=0), -1),
                  (dict(d=0), -1), (dict(pages=0), -1), (dict(page_stride=-8), -1), (dict(k=None), -1),
                  (dict(v=None), -1), (dict(d=12), -2), (dict(d=8), -2), (dict(d=264), -2),
                  (dict(page_size=65537), -2), (dict(pages=1 << 28), -2), (dict(token_stride=124), -3),
                  (dict(head_stride=65), -3), (dict(k=A + 8), -3), (dict(v=A + 2), -3)]


def _rope(cache=None, **changes):
    x = L.QkNormRopeArgs(q=A, k=A, v=A, q_out=2 * A, cache=_cache(**(cache or {})), slots=A, positions=A,
                         cos_sin=A, q_weight=A, k_weight=A, q_stride=512, k_stride=128, v_stride=128,
                         tokens=3, max_positions=100, heads=8, rot=64, interleaved=0, eps=1e-6)
    for k, v in changes.items():
        setattr(x, k, v)
    return x


@pytest.mark.parametrize("changes,status", [
    *[({n: None}, -1) for n in ("q", "k", "v", "q_out", "slots", "positions", "cos_sin")],
    (dict(tokens=-1), -1), (dict(heads=0), -1), (dict(rot=-16), -1), (dict(rot=80), -1),
    (dict(max_positions=-1), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(q_stride=-8), -1), (dict(q_out=A, q_stride=640), -1), (dict(rot=24), -2), (dict(heads=65536), -2),
    (dict(q_stride=516), -3), (dict(k_stride=4), -3), (dict(q=A + 8), -3), (dict(q_weight=A + 4), -3),
    (dict(slots=A + 2), -3), *[(dict(cache=c), s) for c, s in CACHE_REFUSALS], (dict(tokens=0), 0),
])
def test_qk_norm_rope_refusals(lib, changes, status):
    assert lib.lilicorr_qk_norm_rope(ctypes.byref(_rope(**changes)), None) == status


def _attention(cache=None, **changes):
    x = L.AttentionArgs(q=A, out=2 * A, cache=_cache(**(cache or {})), table=A, starts=A, totals=A,
                        workspace=A, workspace_bytes=1 << 40, tokens=5, q_stride=512, N=3, table_width=4,
                        window=0, sinks=0, max_tokens=5, max_length=64, heads=8, causal=1, scale=0.125)
    for k, v in changes.items():
        setattr(x, k, v)
    return x


@pytest.mark.parametrize("changes,status", [
    *[({n: None}, -1) for n in ("q", "out", "table", "starts", "totals")],
    (dict(tokens=-1), -1), (dict(N=0), -1), (dict(table_width=0), -1), (dict(heads=0), -1),
    (dict(heads=7), -1), (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(sinks=3), -1),
    (dict(max_tokens=-1), -1), (dict(max_length=-1), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1),
    (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(out=A), -1),
    (dict(q_stride=-8), -1), (dict(N=(1 << 20) + 1), -2), (dict(tokens=1 << 28), -2),
    (dict(table_width=1 << 27), -2), (dict(cache=dict(pages=1 << 26, page_stride=1 << 39)), -2),
    (dict(q_stride=516), -3), (dict(q=A + 2), -3), (dict(out=A + 8), -3), (dict(table=A + 1), -3),
    (dict(workspace=A + 8), -3), (dict(workspace=None), -4), (dict(workspace_bytes=16), -4),
    *[(dict(cache=c), s) for c, s in CACHE_REFUSALS], (dict(tokens=0), 0), (dict(max_tokens=0), 0),
])
def test_attention_refusals(lib, changes, status):
    assert lib.lilicorr_window_attention(ctypes.byref(_attention(**changes)), None) == status
    both = dict(changes, shared_length=30, shared_table=A)
    if "window" not in changes and "sinks" not in changes:
        assert lib.lilicorr_prefix_attention(ctypes.byref(_attention(**both)), None) == status


def test_which_attention(lib):
    call = lambda f, **c: getattr(lib, f)(ctypes.byref(_attention(**c)), None)  # noqa: E731
    assert call("lilicorr_window_attention", shared_length=30) == -1
    assert call("lilicorr_window_attention", shared_table=A) == -1
    assert call("lilicorr_prefix_attention") == -1
    assert call("lilicorr_prefix_attention", shared_length=30) == -1
    assert call("lilicorr_prefix_attention", shared_length=30, shared_table=A, window=8) == -1
    assert call("lilicorr_prefix_attention", shared_length=30, shared_table=A + 2) == -3


def test_workspace_sizes(lib):
    # many tiles: nothing is split, and a workspace is just its least size
    assert L.lilicorr_window_attention_workspace_bytes(_attention(N=2000, tokens=2000, max_tokens=1)) == 256
    # one request: split keys want room for 32-bit partial results
    one = _attention(N=1, tokens=1, max_tokens=1, table_width=256, max_length=4096)
    need = L.lilicorr_window_attention_workspace_bytes(one)
    assert need > 256 and (need - 256) % (8 * (8 + 64 * 4)) == 0
    assert L.lilicorr_window_attention_workspace_bytes(_attention(heads=7)) == 0
    assert L.lilicorr_prefix_attention_workspace_bytes(_attention()) == 0
    assert L.lilicorr_prefix_attention_workspace_bytes(_attention(shared_length=30)) > 256


def test_python_refusals():
    """The torch conveniences name what is wrong with a tensor."""
    t = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    with pytest.raises(L.LilicorrError, match="lengths|out"):
        L.page_plan(t(2), t(2), t(2, 2), t(2, 4), t(8), t(3, dtype=torch.int64), page_size=4, tokens=3)
    bf = torch.bfloat16
    k = t(4, 8, 2, 64, dtype=bf)
    with pytest.raises(L.LilicorrError, match="cache"):
        L.window_attention(t(3, 4, 64, dtype=bf), k, k, t(1, 4), t(2), t(1))
    with pytest.raises(L.LilicorrError, match="cache"):
        L.qk_norm_rope(t(3, 4, 64, dtype=bf), t(3, 2, 64, dtype=bf), t(3, 2, 64, dtype=bf), t(3), t(3), None,
                       k, k)
