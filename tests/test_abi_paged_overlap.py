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
