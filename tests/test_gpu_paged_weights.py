"""GPU tests that the attentions' weights add up: where every value is 1, every output is exactly 1, however
the scores lie. Each probability is rounded once and the sum is of the rounded ones, so numerator and
denominator differ by fp32 sums alone: n 2^-23 for n keys, 1e-4 at the 900 keys below, while the 16-bit
neighbours of 1 are 2^-8 (bf16) and 2^-11 (fp16) away and the nearer one's middle 2^-9 and 2^-12 = 2.4e-4."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_probabilities_are_rounded_once(lib, d, dtype):
    """A maximum that grows by more than 2^8 between two blocks of one stage, where the block before it has
    powers of almost 2^8 that still weigh the most: keys 64 .. 95 have 2^x, key 100 2^(1.25 x), the rest next
    to nothing, for x in [7, 8)."""
    T, n, P = 128, 128, 16
    q = torch.zeros(T, 1, d, dtype=dtype, device="cuda")
    q[:, 0, 0] = 7 + torch.arange(T, device="cuda") % 32 / 32
    k = torch.zeros(n, d, dtype=dtype, device="cuda")
    k[64:96, 0], k[96:, 0], k[100, 0] = 1.0, -8.0, 1.25
    k = k.view(n // P, P, 1, d)
    table = torch.arange(n // P, dtype=torch.int32, device="cuda")[None]
    ws = lib.window_attention_workspace(q, k, table, causal=False)
    assert ws.numel() == 256  # one chunk
    o = lib.window_attention(q, k, torch.ones_like(k), table, i32([0, T]), i32([n]), causal=False,
                             scale=0.6931471805599453, workspace=ws)
    assert (o == 1).all(), o.float().unique()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new,ctx,shared,window", [([1], [900], 0, 0), ([16, 9], [300, 880], 0, 0),
                                                   ([130], [700], 0, 200), ([7, 40], [90, 300], 500, 0)])
@pytest.mark.parametrize("d", [64, 128, 200])
def test_constant_values_come_out_as_they_are(lib, d, new, ctx, shared, window, dtype):
    """Scores of a standard deviation of up to 16 powers of two."""
    g = torch.Generator().manual_seed(d + len(new))
    P, Hq, Hkv = 16, 4, 2
    totals = [a + b for a, b in zip(new, ctx)]
    width, sp = -(-max(totals) // P), -(-shared // P)
    pages = width * len(new) + sp
    order = torch.randperm(pages, generator=g).to(torch.int32).cuda()
    q = (torch.randn(sum(new), Hq, d, generator=g) * torch.tensor([0.5, 2.0, 8.0, 11.0])[:, None]).to(dtype).cuda()
    k = torch.randn(pages, P, Hkv, d, generator=g).to(dtype).cuda()
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    a = (q, k, torch.ones_like(k))
    b = (order[sp:].view(len(new), width), i32(starts), i32(totals))
    o = lib.prefix_attention(*a, order[:sp], shared, *b) if shared else \
        lib.window_attention(*a, *b, window=window, sinks=3 if window else 0)
    assert (o == 1).all(), o.float().unique()
