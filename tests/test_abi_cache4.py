"""Host-side checks of the 4-bit cache's calls (no GPU): the packed bytes are the C structs' layout, and bad
arguments, sizes, alignments and overlaps are refused before anything is launched."""
import ctypes

import pytest
import torch

import paper_2608_20530_amd as L
from paper_2608_20530_amd import paged4

A = 4096  # a fake, aligned "device" address: never dereferenced on these paths
FAR = 1 << 24  # distances at which no two arguments meet


@pytest.fixture(scope="module")
def lib():
    return L.load_library()


@pytest.mark.parametrize("packer,structure", [(paged4._ROPE, L.QkNormRope4Args), (paged4._ATTENTION, L.Attention4Args),
                                              (paged4._WEIGHTS, L.KeyWeightsArgs), (paged4._EVICT, L.EvictArgs)])
def test_packed_bytes_are_the_struct(packer, structure):
    assert packer.size == ctypes.sizeof(structure)
    count = len(packer.unpack(bytes(packer.size)))
    x = structure.from_buffer_copy(packer.pack(*range(1, count + 1)))
    flat = []
    for name, kind in structure._fields_:
        v = getattr(x, name)
        flat += [getattr(v, n) for n, _ in kind._fields_] if isinstance(v, ctypes.Structure) else [v]
    assert flat == list(range(1, count + 1))


def _make(structure, **values):
    """Every pointer at an address of its own, FAR apart."""
    x = structure(**values)
    at = 1
    for target in (x, x.cache):
        for n, t in type(target)._fields_:
            if t is ctypes.c_void_p:
                setattr(target, n, at * FAR)
                at += 1
    return x


def _change(x, changes):
    for k, v in changes.items():
        target = x.cache if k.startswith("c_") else x
        setattr(target, k.removeprefix("c_"), v)
    return x


def _cache():
    """10 pages of 16 tokens of 2 heads of 64."""
    return L.Cache4Args(page_size=16, heads=2, d=64, pages=10, page_stride=1024, token_stride=64, head_stride=32)


def _rope():
    return _make(L.QkNormRope4Args, cache=_cache(), q_stride=512, k_stride=128, v_stride=128, tokens=5, max_positions=100,
                 dtype=1, heads=8, rot=64, eps=1e-6)


def _attention():
    return _make(L.Attention4Args, cache=_cache(), workspace_bytes=1 << 20, tokens=6, q_stride=512, N=3, table_width=4,
                 max_tokens=6, max_length=64, dtype=1, heads=8, causal=1, scale=0.125)


def _weights():
    return _make(L.KeyWeightsArgs, cache=_cache(), tokens=6, q_stride=512, N=3, table_width=4, max_tokens=6, max_length=64,
                 dtype=1, heads=8, causal=1, scale=0.125, decay=1.0)


def _evict():
    return _make(L.EvictArgs, cache=_cache(), workspace_bytes=1 << 20, N=3, table_width=4, queue_size=10, max_length=64,
                 budget=20, limit=30, sinks=4, recent=8)


CACHE = [(dict(c_page_size=0), -1), (dict(c_heads=0), -1), (dict(c_d=0), -1), (dict(c_pages=0), -1),
         (dict(c_page_stride=-16), -1), (dict(c_token_stride=-16), -1), (dict(c_head_stride=-16), -1),
         (dict(c_k=None), -1), (dict(c_k_scales=None), -1), (dict(c_d=48), -2), (dict(c_d=288), -2),
         (dict(c_page_size=65537), -2), (dict(c_pages=1 << 28), -2), (dict(c_page_stride=1 << 40), -3),
         (dict(c_token_stride=72), -3), (dict(c_head_stride=8), -3), (dict(c_k=FAR + 8), -3), (dict(c_k_scales=FAR + 2), -3)]
VALUES = [(dict(c_v=None), -1), (dict(c_v_scales=None), -1), (dict(c_v=FAR + 8), -3), (dict(c_v_scales=FAR + 1), -3)]
ROWS = [(dict(tokens=-1), -1), (dict(dtype=0), -1), (dict(dtype=3), -1), (dict(heads=0), -1),
        (dict(q_stride=-8), -1), (dict(q_stride=100), -3), (dict(heads=65536), -2)]
STEP = [*ROWS, (dict(N=0), -1), (dict(table_width=0), -1), (dict(max_tokens=-1), -1), (dict(max_length=-1), -1),
        (dict(heads=7), -1), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
        (dict(N=(1 << 20) + 1), -2), (dict(tokens=1 << 28), -2), (dict(table_width=1 << 27), -2),
        (dict(c_token_stride=1 << 27), -2)]


@pytest.mark.parametrize("changes,status", [
    *CACHE, *VALUES, *ROWS, *[({n: None}, -1) for n in ("q", "k", "v", "q_out", "slots", "positions", "cos_sin")],
    (dict(rot=-16), -1), (dict(rot=80), -1), (dict(max_positions=-1), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(k_stride=-8), -1), (dict(v_stride=-8), -1), (dict(rot=8), -2), (dict(tokens=1 << 31), -2), (dict(k_stride=4), -3),
    (dict(v_stride=4), -3), *[({n: FAR + 8}, -3) for n in ("q", "k", "v", "q_out", "cos_sin", "q_weight", "k_weight")],
    (dict(slots=FAR + 2), -3), (dict(positions=FAR + 2), -3)])
def test_qk_norm_rope4_refusals(lib, changes, status):
    assert lib.lilicorr_qk_norm_rope4(ctypes.byref(_change(_rope(), changes)), None) == status


def test_qk_norm_rope4_refuses_overlaps(lib):
    x = _rope()
    for cache_part, last in (("k", 10 * 1024 - 16), ("v", 10 * 1024 - 16), ("k_scales", 636), ("v_scales", 636)):
        at = getattr(x.cache, cache_part)
        for name in ("q", "k", "v", "q_out"):
            size = 5120 if name in ("q", "q_out") else 1280  # 5 tokens of 8 or 2 heads of 64, 2 bytes
            for a in (at, at + last // 16 * 16, at - size + 16):
                assert lib.lilicorr_qk_norm_rope4(ctypes.byref(_change(_rope(), {name: a})), None) == -1, (cache_part, name)
    for name, size in (("q", 5120), ("k", 1280), ("v", 1280)):
        for a in (x.q_out + 16, x.q_out - size + 16, x.q_out + 5120 - 16):
            assert lib.lilicorr_qk_norm_rope4(ctypes.byref(_change(_rope(), {name: a})), None) == -1
    assert lib.lilicorr_qk_norm_rope4(ctypes.byref(_change(_rope(), dict(q=x.q_out, q_stride=520))), None) == -1


@pytest.mark.parametrize("changes,status", [
    *CACHE, *VALUES, *STEP, *[({n: None}, -1) for n in ("q", "out", "table", "starts", "totals")],
    (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(sinks=4), -1),
    *[({n: FAR + 8}, -3) for n in ("q", "out", "workspace")],
    *[({n: FAR + 2}, -3) for n in ("lse", "table", "starts", "totals")],
    (dict(workspace=None), -4), (dict(workspace_bytes=255), -4)])
def test_attention4_refusals(lib, changes, status):
    assert lib.lilicorr_window_attention4(ctypes.byref(_change(_attention(), changes)), None) == status


def test_attention4_refuses_overlaps(lib):
    row = 8 * 64 * 2
    read = {"q": 6 * row, "table": 48, "starts": 16, "totals": 12, "c_k": 10240, "c_v": 10240, "c_k_scales": 640,
            "c_v_scales": 640}
    need = L.lilicorr_window_attention4_workspace_bytes(_attention())
    written = {"out": 6 * row, "lse": 6 * 8 * 4, "workspace": need}
    place = lambda x, n: getattr(x.cache, n[2:]) if n.startswith("c_") else getattr(x, n)  # noqa: E731
    for w, size in written.items():
        for r, bytes_ in {**read, **written}.items():
            if r == w:
                continue
            at = place(_attention(), r)
            for a in (at, at + (bytes_ - 1) // 16 * 16, at - (size - 1) // 16 * 16):
                assert lib.lilicorr_window_attention4(ctypes.byref(_change(_attention(), {w: a})), None) == -1, (w, r, a - at)


def test_attention4_workspace_sizes():
    need = lambda **kw: L.lilicorr_window_attention4_workspace_bytes(_change(_attention(), kw))  # noqa: E731
    assert need() == 256  # 64 keys at most: nothing is split
    split = dict(table_width=1000, max_length=16000, tokens=3, max_tokens=1)
    assert need(**split) > 3 * 8 * (16 + 64 * 4)
    assert need(**split, q=None, out=None, c_k=None, workspace=None) == need(**split)  # pointers are not looked at
    for bad, _ in STEP[:2] + CACHE[:4]:
        assert need(**bad) == 0
    for far in (1 << 31, 1 << 62, (1 << 63) - 1):  # windows and sinks that stand for "without end"
        long = dict(split, window=far, sinks=far)
        assert need(**long) == need(**split)


@pytest.mark.parametrize("changes,status", [
    *CACHE, *STEP, *[({n: None}, -1) for n in ("q", "lse", "weights", "table", "starts", "totals")],
    (dict(decay=-0.5), -1), (dict(decay=float("nan")), -1), (dict(decay=float("inf")), -1),
    *[({n: FAR + 8}, -3) for n in ("q", "weights")], *[({n: FAR + 2}, -3) for n in ("lse", "table", "starts", "totals")],
    (dict(N=1 << 20, table_width=1 << 22, max_length=1 << 26), -2)])
def test_key_weights_refusals(lib, changes, status):
    assert lib.lilicorr_key_weights(ctypes.byref(_change(_weights(), changes)), None) == status


def test_key_weights_refuses_overlaps(lib):
    size = 10 * 2 * 16 * 4
    read = {"q": 6 * 1024, "lse": 6 * 8 * 4, "table": 48, "starts": 16, "totals": 12, "c_k": 10240, "c_k_scales": 640}
    for r, bytes_ in read.items():
        x = _weights()
        at = getattr(x.cache, r[2:]) if r.startswith("c_") else getattr(x, r)
        for a in (at, at + (bytes_ - 1) // 16 * 16, at - (size - 1) // 16 * 16):
            assert lib.lilicorr_key_weights(ctypes.byref(_change(_weights(), dict(weights=a))), None) == -1, (r, a - at)


EVICT_POINTERS = ("weights", "table", "totals", "pages", "queue", "cursor", "totals_out", "pages_out", "evicted", "cursor_out")


@pytest.mark.parametrize("changes,status", [
    *[c for c in CACHE if "c_token_stride" not in c[0] or c[1] != -2], *VALUES, *[({n: None}, -1) for n in EVICT_POINTERS],
    (dict(N=0), -1), (dict(table_width=0), -1), (dict(queue_size=0), -1), (dict(max_length=-1), -1), (dict(budget=0), -1),
    (dict(limit=19), -1), (dict(sinks=-1), -1), (dict(recent=-1), -1), (dict(sinks=12, recent=9), -1),
    (dict(sinks=1 << 62, recent=1 << 62), -1), (dict(N=4097), -2), (dict(table_width=1 << 27), -2),
    (dict(queue_size=1 << 31), -2), (dict(budget=(1 << 30) + 1, limit=1 << 31), -2),
    *[({n: FAR + 2}, -3) for n in EVICT_POINTERS], (dict(cursor=FAR + 4), -3), (dict(cursor_out=FAR + 4), -3),
    (dict(weights=FAR + 8), -3), (dict(workspace=FAR + 8), -3), (dict(workspace=None), -4), (dict(workspace_bytes=255), -4)])
def test_evict_refusals(lib, changes, status):
    assert lib.lilicorr_evict(ctypes.byref(_change(_evict(), changes)), None) == status


def test_evict_refuses_overlaps(lib):
    sizes = {"totals": 12, "pages": 24, "cursor": 24, "table": 48, "queue": 40, "totals_out": 12, "pages_out": 24,
             "evicted": 12, "cursor_out": 24, "weights": 1280, "workspace": 480, "c_k": 10240, "c_v": 10240,
             "c_k_scales": 640, "c_v_scales": 640}
    read = ("totals", "pages", "cursor", "table")
    assert L.lilicorr_evict_workspace_bytes(_evict()) == sizes["workspace"]
    for one in sizes:
        for other in sizes:
            if one == other or (one in read and other in read) or (one[:2] == "c_" and other[:2] == "c_"):
                continue
            x = _evict()
            at = getattr(x.cache, other[2:]) if other[:2] == "c_" else getattr(x, other)
            for a in (at, at + (sizes[other] - 1) // 16 * 16):
                assert lib.lilicorr_evict(ctypes.byref(_change(_evict(), {one: a})), None) == -1, (one, other, a - at)


def test_evict_workspace_sizes():
    need = lambda **kw: L.lilicorr_evict_workspace_bytes(_change(_evict(), kw))  # noqa: E731
    assert need() == 3 * 2 * 20 * 4
    assert need(budget=64, limit=64) == 256  # no request can be longer
    assert need(budget=0) == need(N=5000) == need(c_d=48) == 0


def test_nothing_to_do(lib):
    """No tokens: no pointer is looked at."""
    none = dict.fromkeys(("q", "table", "starts", "totals"))
    assert lib.lilicorr_window_attention4(ctypes.byref(_change(_attention(), dict(none, tokens=0, out=None))), None) == 0
    assert lib.lilicorr_key_weights(ctypes.byref(_change(_weights(), dict(none, tokens=0, weights=None))), None) == 0
    assert lib.lilicorr_qk_norm_rope4(ctypes.byref(_change(_rope(), dict(tokens=0, q=None, slots=None))), None) == 0
    for name in ("qk_norm_rope4", "window_attention4", "key_weights", "evict"):
        assert getattr(lib, "lilicorr_" + name)(None, None) == -1
    assert lib.lilicorr_window_attention4_workspace_bytes(None) == lib.lilicorr_evict_workspace_bytes(None) == 0


def test_python_refusals():
    """Host tensors, types and shapes are refused by the binding."""
    cache = L.cache4(4, 16, 2, 64, device="cpu")
    assert cache.k.shape == (4, 16, 2, 32) and cache.k_scales.shape == (4, 16, 2, 2) and (cache.k_scales == 1).all()
    with pytest.raises(L.LilicorrError, match="blocks of 32"):
        L.cache4(4, 16, 2, 48, device="cpu")
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    ints = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros(3, 4, dtype=torch.int32)
    for call in (lambda: L.qk_norm_rope4(q, q[:, :2], q[:, :2], ints[:3], ints[:3], None, cache),
                 lambda: L.window_attention4(q, cache, table, ints, ints[:3]),
                 lambda: L.window_attention4_workspace(q, cache, table),
                 lambda: L.key_weights(q, torch.zeros(3, 8), cache, table, ints, ints[:3], torch.zeros(4, 2, 16)),
                 lambda: L.evict(cache, torch.zeros(4, 2, 16), table, ints[:3], torch.zeros(3, 2, dtype=torch.int32),
                                 ints, torch.zeros(3, dtype=torch.int64), budget=20)):
        with pytest.raises(L.LilicorrError, match="device tensors"):
            call()
