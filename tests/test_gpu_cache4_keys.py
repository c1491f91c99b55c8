"""GPU tests of keys whose squares, sums or products leave the range of fp32: codes and scales are those of the arithmetic in
64 bits all the same, equal to the definition's."""
import numpy as np
import pytest
import torch

from test_gpu_cache4 import BF, check_write, host, i32, make_cache

pytestmark = pytest.mark.gpu

ENDS = [-133, -120, -96, -75, -72, -70, -67, -66, -64, -63, -61, -50, -30, 20, 29, 31, 50, 59, 60, 61, 62, 63, 64, 90, 110, 126]


def write(lib, k, eps, rot, inter, weight, seed=0):
    """Keys k [T, heads, d] with ordinary queries and values, checked."""
    T, heads, d = k.shape
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(T, heads, d, generator=g).to(BF).cuda()
    cache = make_cache(lib, T // 8 + 2, 8, heads, d)
    before = [np.ascontiguousarray(host(y)) for y in cache]
    slots, positions = i32(list(range(T))), i32([7 * t % 5000 for t in range(T)])
    ang = torch.rand(5000, max(rot // 2, 1), generator=g, dtype=torch.float64)[:, :rot // 2] * 6.3
    cs = torch.cat((ang.cos(), ang.sin()), 1).float().cuda() if rot else None
    w = [None, weight.cuda()]
    out = lib.qk_norm_rope4(q, k.cuda(), q, slots, positions, cs, cache, k_weight=w[1], eps=eps, interleaved=inter)
    torch.cuda.synchronize()
    check_write(q, k, q, slots, positions, cs, cache, w, out, before, BF, rot, inter, eps=eps)
    assert not (host(cache.k_scales).reshape(-1, *cache.k_scales.shape[2:])[:T] == 255).any()


@pytest.mark.parametrize("d,heads,rot,inter", [(128, 2, 128, False), (64, 3, 64, True), (96, 1, 32, False), (256, 1, 0, False)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_keys_of_every_size(lib, d, heads, rot, inter, eps):
    print("keys", d, heads, rot, inter, eps, flush=True)
    g = torch.Generator().manual_seed(3)
    rows = [torch.randn(heads, d, generator=g).clamp(-3, 3) * 2.0 ** min(e, 60) * 2.0 ** max(e - 60, 0) for e in ENDS]
    rows += [torch.full((heads, d), 2.0 ** 61), torch.full((heads, d), -(2.0 ** 64)), torch.full((heads, d), 2.0 ** -66)]
    k = torch.stack(rows).to(BF)
    k[k == 0] = 2.0 ** -133  # (a head of zeros has no norm without eps)
    write(lib, k, eps, rot, inter, 1 + 0.2 * torch.randn(d, generator=g))


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (0, False)])
def test_sizes_side_by_side(lib, rot, inter):
    """Within a head blocks of very different sizes, and weights that bring them up or down."""
    d, T = 64, 64
    g = torch.Generator().manual_seed(4)
    k = torch.randn(T, 2, d, generator=g)
    for t in range(T):
        a, b = ENDS[t % len(ENDS)], ENDS[(7 * t + 3) % len(ENDS)]
        k[t, :, :32] *= 2.0 ** (min(a, 60))
        k[t, :, 32:] *= 2.0 ** (min(b, 60))
        k[t, 1, ::5] = 0
    for kind in range(3):
        weight = 1 + 0.2 * torch.randn(d, generator=g)
        if kind == 1:
            weight[::3] *= 2.0 ** 40
        elif kind == 2:
            weight[1::4] *= 2.0 ** -40
        write(lib, k.to(BF), 1e-6, rot, inter, weight, seed=kind)


def test_keys_without_a_norm(lib):
    d, T = 64, len(ENDS)
    g = torch.Generator().manual_seed(5)
    k = torch.stack([torch.randn(2, d, generator=g).clamp(-1.5, 1.5) * 2.0 ** min(e, 60) * 2.0 ** max(e - 60, 0) for e in ENDS]).to(BF)
    q = torch.randn(T, 2, d, generator=g).to(BF).cuda()
    for rot in (0, 64):
        cache = make_cache(lib, T // 8 + 2, 8, 2, d)
        before = [np.ascontiguousarray(host(y)) for y in cache]
        slots, positions = i32(list(range(T))), i32([3 * t for t in range(T)])
        ang = torch.rand(5000, 32, generator=g, dtype=torch.float64) * 6.3
        cs = torch.cat((ang.cos(), ang.sin()), 1).float().cuda() if rot else None
        out = lib.qk_norm_rope4(q, k.cuda(), q, slots, positions, cs, cache)
        torch.cuda.synchronize()
        check_write(q, k, q, slots, positions, cs, cache, (None, None), out, before, BF, rot, False)
