"""Host-side checks (no GPU) of how far the attentions split their keys, by the size of the workspace: the 128-row
kernels of heads of up to 128 run two workgroups a compute unit, 512 at once."""
import pytest

import paper_2608_20530_amd as L

A = 4096  # an address that nothing reads


def _chunks(N, d, keys):
    """N requests of 128 rows against `keys` keys, one head: a tile a request."""
    cache = L.Cache(k=A, v=A, dtype=1, page_size=64, heads=1, d=d, pages=1000, page_stride=64 * d, token_stride=d,
                    head_stride=0)
    need = L.lilicorr_window_attention_workspace_bytes(L.AttentionArgs(
        q=A, out=A, cache=cache, table=A, starts=A, totals=A, tokens=N * 128, q_stride=d, N=N,
        table_width=keys // 64, max_tokens=128, max_length=keys, heads=1, causal=0, scale=0.1))
    assert need >= 256
    return max((need - 256) // (N * 128 * (8 + 4 * d)), 1)


@pytest.mark.parametrize("d", [24, 64, 72, 96, 120, 128])
def test_tiles_fill_the_chip_twice(d):
    L.load_library()
    for keys in (4096, 16384, 65536):
        assert _chunks(256, d, keys) == 2  # one tile a compute unit: two halves
        assert _chunks(512, d, keys) == 1  # all at once
    assert _chunks(704, d, 16384) > 1      # whole, they would leave the second round mostly empty
    assert _chunks(768, d, 65536) > 1
