"""GPU tests that run every attention kernel: head widths of each kind (64, 128 and 256, below each, and 65 to 96)
in both types at each tile height, and chunks that are longer than the page numbers a wave keeps, so that it
fetches more of them, with the first tokens and missing pages among them. Inputs, definition and tolerances
are those of test_gpu_paged.py."""
import pytest
import torch

from test_gpu_paged import BF, HF, _attend, _attention_inputs, _check, _want, i32

pytestmark = pytest.mark.gpu

# new tokens and those before them; with three query heads to a key head their rows fit 32, 64 and 128
ROWS = {32: ([5, 1], [150, 61]), 64: ([16, 3], [150, 61]), 128: ([40, 23], [150, 61])}
MASKS = {"window": dict(window=70, sinks=5), "all": dict(causal=False), "prefix": dict(shared=90)}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [16, 24, 56, 64, 72, 96, 104, 120, 128, 136, 248, 256])
def test_every_kernel(lib, d, dtype, rows, mask):
    print("attention", d, dtype, rows, mask, flush=True)
    new, ctx = ROWS[rows]  # (a shared prefix's tiles hold all requests' rows)
    kw = dict(MASKS[mask])
    shared = kw.pop("shared", 0)
    x = _attention_inputs(new, ctx, 6, 2, d, 24, dtype, shared=shared, seed=d)
    _check(x, _attend(lib, x, shared, max_tokens=max(new), max_length=int(x["totals"].max()), **kw),
           _want(x, shared, **kw))


# the first tokens' pages, the window's, and the tokens whose page is missing, by position
LONG = {"window": (dict(window=700, sinks=7), ()), "window, missing": (dict(window=700, sinks=7), (1300, 1301, 1390)),
        "many sinks, missing": (dict(window=300, sinks=400), (3, 333, 1290)), "all": (dict(), ()),
        "all, missing": (dict(causal=False), (0, 256, 700, 1023, 1400))}


@pytest.mark.parametrize("case", LONG)
@pytest.mark.parametrize("rows,T", [(32, 3), (64, 12), (128, 30)])
@pytest.mark.parametrize("d,dtype", [(64, HF), (96, BF), (128, BF), (256, HF)])
def test_more_pages_than_a_wave_keeps(lib, d, dtype, rows, T, case):
    """Pages of one token. Hundreds of requests with the same tokens, so that the keys are hardly split; each
    has the same result, and the first one's is compared with the definition."""
    print("page numbers", d, rows, case, flush=True)
    mask, gone = LONG[case]
    total, Hq, N = 1400 + T, 4, 700
    x = _attention_inputs([T], [1400], Hq, 1, d, 1, dtype, seed=rows)
    for j in gone:
        x["table"][0, j] = -1 if j % 2 else x["k_cache"].shape[0]
    y = dict(x, q=x["q"].repeat(N, 1, 1), table=x["table"].repeat(N, 1), starts=i32(range(0, N * T + 1, T)),
             totals=i32([total] * N))
    kw = dict(mask, max_tokens=T, max_length=total)
    ws = lib.window_attention_workspace(y["q"], y["k_cache"], y["table"], **kw)
    parts = max((ws.numel() - 256) // (N * T * Hq * (8 + 4 * d)), 1)
    assert 707 // parts > 256, "the chunks are too short for this test"
    got = _attend(lib, y, workspace=ws, **kw).view(N, T, Hq, d)
    assert (got == got[:1]).all()
    _check(x, got[0], _want(x, **mask))


def test_windows_without_end(lib):
    x = _attention_inputs([16, 1], [300, 90], 4, 2, 64, 16, BF)
    want = _attend(lib, x)
    for far in (1 << 30, 1 << 62, (1 << 63) - 1):
        assert torch.equal(_attend(lib, x, window=far), want)
        assert torch.equal(_attend(lib, x, window=far, sinks=far), want)
    _check(x, want, _want(x))
