"""Host-side checks (no GPU): windows and sinks that stand for "without end" make the plan of the largest ones
that a sequence can have, whatever 64-bit value stands for it."""
import pytest

import paper_2608_20530_amd as L

A, LONG = 4096, 1 << 30  # an address that nothing reads; the longest sequences have 2^30 tokens


def _bytes(window, sinks, causal, N, tokens, max_tokens):
    cache = L.Cache(k=A, v=A, dtype=1, page_size=16, heads=2, d=64, pages=1000, page_stride=2048, token_stride=128,
                    head_stride=64)
    return L.lilicorr_window_attention_workspace_bytes(L.AttentionArgs(
        q=A, out=2 * A, cache=cache, table=A, starts=A, totals=A, tokens=tokens, q_stride=512, N=N,
        table_width=256, window=window, sinks=sinks, max_tokens=max_tokens, max_length=4096, heads=8,
        causal=causal, scale=0.125))


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("N,tokens,max_tokens", [(1, 64, 64), (3, 5, 4), (1, 1, 1)])
@pytest.mark.parametrize("far", [LONG + 1, 1 << 31, 1 << 32, 1 << 62, (1 << 63) - 65, (1 << 63) - 1])
def test_far_windows_and_sinks(far, N, tokens, max_tokens, causal):
    L.load_library()
    rest = (causal, N, tokens, max_tokens)
    want = _bytes(LONG, LONG, *rest)
    assert want > 256  # long sequences of few requests are split
    assert _bytes(far, far, *rest) == want
    assert _bytes(far, 0, *rest) == _bytes(LONG, 0, *rest) == want
    assert _bytes(32, far, *rest) == _bytes(32, LONG, *rest) == want
