"""GPU tests of the 4-bit attention with scores so large (2^24 powers of two and more) that rounding the scaled score
alone exceeds what the running maximum lets pass. Keys of one size throughout have equal scores, whatever is
rounded, so the output is the mean of the values that share the largest one; tolerances of ordinary rows are those of
test_gpu_cache4.py. A far row's logarithm is known to 2^-24 (d + 6) of the score (fp32 sums of d products, the scale's and
the logarithm's roundings)."""
import numpy as np
import pytest
import torch

from test_gpu_cache4 import BF, HF, P_U, U, attend, attention_inputs, check_attention, f64, host, values, wanted, widened

pytestmark = pytest.mark.gpu

CASES = [
    # new, ctx, Hq, Hkv, d, page, dtype, N, keys: rings of one wave's own, shared ones, registers
    ([1], [700], 8, 2, 128, 16, BF, 1, 720),
    ([16], [300], 8, 2, 64, 16, HF, 1, 400),
    ([90], [50], 4, 1, 128, 16, BF, 1, 160),
    ([7], [90], 4, 2, 256, 16, BF, 1, 128),
    ([1], [900], 16, 4, 128, 16, BF, 64, 8192),
    ([16], [500], 16, 4, 128, 16, HF, 64, 8192),
    ([8], [300], 8, 2, 128, 24, HF, 1, 336),
    ([40], [70], 6, 2, 96, 16, BF, 1, 128),
]


@pytest.mark.parametrize("new,ctx,Hq,Hkv,d,page,dtype,N,keys", CASES)
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores(lib, new, ctx, Hq, Hkv, d, page, dtype, N, keys, sign):
    """Every third row is 20480 throughout, the others are ordinary. Keys: the last third of the context 6144 throughout, every
    seventh of them 4096, the others ordinary. With the other sign rows are -20480 and all keys large, so that every
    score is far below zero."""
    print("far scores", new, ctx, Hq, Hkv, d, page, dtype, sign, flush=True)
    x = attention_inputs(lib, new, ctx, Hq, Hkv, d, page, dtype)
    T, total = new[0], new[0] + ctx[0]
    row, c = host(x["table"])[0], x["cache"]
    large = range(total - T - ctx[0] // 3, total - T) if sign > 0 else range(total)
    for j in large:
        c.k[row[j // page], j % page] = 0x66 if j % 7 == 0 else 0x77  # 4 or 6
        c.k_scales[row[j // page], j % page] = 127 + 10
    far = torch.zeros(T, Hq, dtype=torch.bool)
    far.view(-1)[::3] = True
    # queries of ordinary rows small, so that their scores stay ordinary beside such keys
    x["q"] = torch.where(far.cuda()[..., None], sign * 20480.0, x["q"].float() * 2.0 ** -12).to(dtype)
    out, lse = attend(lib, widened(x, N, keys), max_tokens=T, max_length=keys)
    near = dict(x, q=torch.where(far.cuda()[..., None], 0.0, x["q"].float()).to(dtype))
    want = wanted(near)
    ok = ~far.numpy()
    exact = [np.where(ok.reshape(T, Hq, *[1] * (w.ndim - 2)), w, 0) if w.ndim > 1 else w for w in want]
    check_attention(near, (torch.where(far.cuda()[..., None], 0.0, out.float()).to(dtype),
                           torch.where(far.cuda(), 0.0, lse)), (*exact[:4], np.where(ok, want[4], 0)))
    k, v = values(c)
    k = np.array([k[row[j // page], j % page] for j in range(total)])
    v = np.array([v[row[j // page], j % page] for j in range(total)])
    for t, h in np.argwhere(far.numpy()):
        kv, seen = h // (Hq // Hkv), total - T + t + 1
        s = sign * 20480.0 * k[:seen, kv].sum(-1) / np.sqrt(d)
        best = s == s.max()  # others are farther away than any power counts
        assert (s[~best] < s.max() - 1000).all()
        exact, size = v[:seen, kv][best].mean(0), np.abs(v[:seen, kv][best]).mean(0)
        tol = U[dtype] * np.abs(exact) + (P_U[dtype] + best.sum() * 2.0 ** -23) * size + (2.0 ** -25 if dtype == HF else 0)
        assert (np.abs(f64(out[t, h]) - exact) <= tol).all(), (t, h)
        assert abs(float(lse[t, h]) - s.max()) <= 2.0 ** -24 * (d + 6) * np.abs(20480.0 * k[:seen, kv]).sum(-1).max() / np.sqrt(d)
