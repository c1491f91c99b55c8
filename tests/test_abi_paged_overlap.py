"""Host-side checks (no GPU): paged-cache calls whose outputs lie on what other workgroups still read are
refused before anything is launched."""
import ctypes

import pytest

import paper_2608_20530_amd as L

INVALID = -1
N, M, C, T = 4, 8, 64, 10
BYTES = {"lengths": 4 * N, "incoming": 4 * N, "pages": 8 * N, "table": 4 * N * M, "queue": 4 * C, "cursor": 24,
         "pages_out": 8 * N, "cursor_out": 24, "starts": 4 * (N + 1), "totals": 4 * N, "slots": 4 * T,
         "positions": 4 * T}
READ = ("lengths", "incoming", "pages", "cursor")


@pytest.fixture(scope="module")
def lib():
    return L.load_library()


def _plan(**changes):
    """Arguments at addresses of their own, 4096 bytes apart, that nothing on these paths reads."""
    x = L.PagePlanArgs(**{n: 4096 * (i + 1) for i, n in enumerate(BYTES)}, N=N, page_size=16, table_width=M,
                       queue_size=C, tokens=T, window=0, sinks=0)
    for k, v in changes.items():
        setattr(x, k, v)
    return x


@pytest.mark.parametrize("one,other", [(a, b) for a in BYTES for b in BYTES
                                       if a != b and not (a in READ and b in READ)])
def test_page_plan_refuses_overlaps(lib, one, other):
    at = getattr(_plan(), other)
    assert lib.lilicorr_page_plan(ctypes.byref(_plan(**{one: at})), None) == INVALID
    align = 8 if "cursor" in one else 4
    last = (at + BYTES[other] - 1) // align * align  # the last place in it that `one` may begin at
    assert lib.lilicorr_page_plan(ctypes.byref(_plan(**{one: last})), None) == INVALID


def _rope(**changes):
    """3 tokens of 8 + 2 x 2 heads of 64: rows of 1536 bytes in one projection's output at 4096."""
    cache = L.Cache(k=1 << 20, v=1 << 21, dtype=1, page_size=16, heads=2, d=64, pages=10, page_stride=2048,
                    token_stride=128, head_stride=64)
    x = L.QkNormRopeArgs(q=4096, k=4096 + 1024, v=4096 + 1280, q_out=1 << 16, cache=cache, slots=1 << 17,
                         positions=1 << 18, cos_sin=1 << 19, q_stride=768, k_stride=768, v_stride=768, tokens=3,
                         max_positions=100, heads=8, rot=64, interleaved=0, eps=1e-6)
    for k, v in changes.items():
        setattr(x, k, v)
    return x


@pytest.mark.parametrize("q_out", [4096 - 3072 + 16, 4096 + 16, 4096 + 1024, 4096 + 1280, 4096 + 2 * 1536 + 1024 - 16,
                                   4096 + 2 * 1536 + 1280, 4096 + 3 * 1536 - 16])
def test_qk_norm_rope_refuses_overlaps(lib, q_out):
    """q_out is 3072 bytes; it may be q itself, and nothing else that the call reads row by row."""
    assert lib.lilicorr_qk_norm_rope(ctypes.byref(_rope(q_out=q_out)), None) == INVALID
    if q_out > 3072:  # k and v in places of their own that q_out meets the last row of
        for name in ("k", "v"):
            at = q_out - 2 * 1536
            rest = {n: 1 << 22 for n in ("q", "k", "v") if n != name}
            assert lib.lilicorr_qk_norm_rope(ctypes.byref(_rope(q_out=q_out, **{name: at}, **rest)), None) == INVALID


@pytest.mark.parametrize("out", [4096 + 16, 4096 + 1024, 4096 + 1536, 4096 + 2 * 1536 + 1024 - 16, 4096 - 3072 + 16])
@pytest.mark.parametrize("name", ["lilicorr_window_attention", "lilicorr_prefix_attention"])
def test_attention_refuses_overlaps(lib, name, out):
    """q: 3 rows of 1024 bytes, 1536 apart; out: 3072 bytes."""
    prefix = dict(shared_table=1 << 18, shared_length=30) if "prefix" in name else {}
    x = L.AttentionArgs(q=4096, out=out, cache=_rope().cache, table=1 << 17, starts=1 << 17, totals=1 << 17,
                        workspace=1 << 22, workspace_bytes=1 << 40, tokens=3, q_stride=768, N=3, table_width=4,
                        max_tokens=3, max_length=64, heads=8, causal=1, scale=0.125, **prefix)
    assert getattr(lib, name)(ctypes.byref(x), None) == INVALID
