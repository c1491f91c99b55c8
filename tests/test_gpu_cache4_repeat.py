"""GPU tests: the 4-bit attention gives the same bits in every launch where partial results of many rows are joined. A launch
with an error here was one of three to ten, a row at a time, with fresh outputs and used ones."""
import pytest
import torch

from test_gpu_cache4 import BF, HF, attend, attention_inputs, widened

pytestmark = pytest.mark.gpu

CASES = [
    # new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype, keys
    ([33 - 5 * n % 34 for n in range(37)], [17 + 400 * n % 3000 for n in range(37)], 14, 2, 64, 24, 1000, 7, False, HF, 3120),
    ([16] * 64, [200 + 11 * n for n in range(64)], 32, 8, 128, 16, 0, 0, True, BF, 16384),
    ([1] * 128, [100 + 6 * n for n in range(128)], 32, 8, 128, 16, 0, 0, True, HF, 16384),
    ([9] * 40, [50 + 20 * n for n in range(40)], 8, 4, 256, 16, 0, 0, True, BF, 8192),
]


@pytest.mark.parametrize("new,ctx,Hq,Hkv,d,page,window,sinks,causal,dtype,keys", CASES)
def test_launches_repeat(lib, new, ctx, Hq, Hkv, d, page, window, sinks, causal, dtype, keys):
    print("repeat", len(new), Hq, Hkv, d, page, window, dtype, flush=True)
    x = widened(attention_inputs(lib, new, ctx, Hq, Hkv, d, page, dtype), len(new), keys)
    bounds = dict(window=window, sinks=sinks, causal=causal, max_tokens=max(new), max_length=keys)
    space = lib.window_attention4_workspace(x["q"], x["cache"], x["table"], **bounds)
    rows = x["q"].shape[0] * Hq
    assert space.numel() > 2 * rows * 4 * d and rows > 1024  # several partial results a row, and many rows
    want = attend(lib, x, **bounds)
    for launch in range(40):
        if launch % 2:
            space.fill_(launch)
        got = attend(lib, x, **bounds, workspace=space)
        same = [torch.equal(a, b) for a, b in zip(got, want)]
        assert same == [True, True], (launch, (got[0] != want[0]).nonzero()[:3].tolist())
