"""A 4-bit cache without the parts that a call reads is refused by the binding (no GPU), in every call's own error."""
import pytest
import torch

import paper_2608_20530_amd as L

WHOLE = L.cache4(4, 16, 2, 64, device="cpu")
Q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
INTS, TABLE = torch.zeros(4, dtype=torch.int32), torch.zeros(3, 4, dtype=torch.int32)
CALLS = {
    "qk_norm_rope4": lambda c: L.qk_norm_rope4(Q, Q[:, :2], Q[:, :2], INTS[:3], INTS[:3], None, c),
    "window_attention4": lambda c: L.window_attention4(Q, c, TABLE, INTS, INTS[:3]),
    "window_attention4 with a workspace": lambda c: L.window_attention4(Q, c, TABLE, INTS, INTS[:3], workspace=INTS),
    "window_attention4_workspace": lambda c: L.window_attention4_workspace(Q, c, TABLE),
    "evict": lambda c: L.evict(c, torch.zeros(4, 2, 16), TABLE, INTS[:3], torch.zeros(3, 2, dtype=torch.int32), INTS,
                               torch.zeros(3, dtype=torch.int64), budget=20),
    "evict_workspace": lambda c: L.evict_workspace(c, TABLE, budget=20),
    "key_weights": lambda c: L.key_weights(Q, torch.zeros(3, 8), c, TABLE, INTS, INTS[:3], torch.zeros(4, 2, 16)),
}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("missing", WHOLE._fields)
def test_parts_that_are_missing(call, missing):
    cache = WHOLE._replace(**{missing: None})
    needed = missing in ("k", "k_scales") or call != "key_weights"
    # without values key_weights comes as far as the next thing that is wrong here: host memory
    workspace = "must be a contiguous device tensor"
    with pytest.raises(L.LilicorrError, match=f"needs the cache's keys|{workspace}" if needed else "device tensors"):
        CALLS[call](cache)
