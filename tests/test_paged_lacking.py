"""Steps after one in which the queue of free pages ran out: tokens that got no page were stored nowhere, so
their request goes on without them, and what the pages that it gets later held before is never read as keys.
Tolerances as in test_gpu_paged.py: u for the output and u sum p|v| for the probabilities (u = 2^-8), fp32
scores and sums 1e-5."""
import numpy as np
import pytest
import torch

import oracle.paged as ref

I32 = dict(dtype=torch.int32, device="cuda")


def test_page_plan_after_lacking_by_hand():
    # 13 tokens on pages of 4, two pages there: 8 are stored, entries 2 and 3 have none
    table = np.full((1, 6), -1, np.int32)
    one = ref.page_plan([0], [13], [(0, 0)], table, np.array([5, 3, 9, 9], np.int32), [0, 2, 0], 4, 13)
    assert one["pages"].tolist() == [[2, 0]] and one["totals"].tolist() == [13] and one["cursor"][2] == 2
    assert one["slots"].tolist() == [20, 21, 22, 23, 12, 13, 14, 15] + [-1] * 5
    # two pages come back; the next token is token 8, not 13
    queue = np.array([5, 3, 7, 1], np.int32)
    two = ref.page_plan(one["totals"], [2], one["pages"], one["table"], queue, [2, 4, 0], 4, 2)
    assert two["positions"].tolist() == [8, 9] and two["slots"].tolist() == [28, 29]
    assert two["totals"].tolist() == [10] and two["pages"].tolist() == [[3, 0]]
    assert two["table"].tolist() == [[5, 3, 7, -1, -1, -1]]


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 3)])
def test_keys_that_were_never_written_are_never_read(lib, window, sinks):
    """Request 0 runs out of pages in the middle of a prompt, tries again in vain, and goes on when request 1
    has ended. The cache is full of large values of earlier owners. Every step's plan is the definition's, and
    its attention that over the tokens that were stored."""
    P, M, d, Hkv, Hq, pages = 8, 12, 64, 2, 4, 11
    g = torch.Generator().manual_seed(3)
    kc = torch.full((pages, P, Hkv, d), 30.0, dtype=torch.bfloat16, device="cuda")
    vc = torch.full_like(kc, 1000.0)
    free = [4, 0, 10, 7, 2]
    table = torch.full((2, M), -1, **I32)
    queue = torch.tensor(free + [-9] * (pages - len(free)), **I32)
    cursor = torch.tensor([0, len(free), 0], device="cuda")
    lengths, held = torch.zeros(2, **I32), torch.zeros(2, 2, **I32)
    kept = [[torch.zeros(0, Hkv, d, dtype=torch.float64)] * 2 for _ in range(2)]
    for step, (new, stored, lacking) in enumerate([((20, 14), (20, 14), 0), ((19, 1), (4, 1), 2),
                                                   ((5, -1), (0, -1), 1), ((8, 0), (8, 0), 0),
                                                   ((0, 3), (0, 3), 0)]):
        counts = [max(n, 0) for n in new]
        T = sum(counts)
        r = lambda h: torch.randn(T, h, d, generator=g).to(torch.bfloat16).cuda()  # noqa: E731,B023
        q, k, v = r(Hq), r(Hkv), r(Hkv)
        incoming = torch.tensor(new, **I32)
        host = [t.cpu().numpy() for t in (lengths, incoming, held, table, queue, cursor)]
        plan = lib.page_plan(lengths, incoming, held, table, queue, cursor, page_size=P, tokens=T,
                             window=window, sinks=sinks)
        want = ref.page_plan(*host, P, T, window, sinks)
        for name in plan._fields:
            assert np.array_equal(getattr(plan, name).cpu().numpy(), want[name]), (step, name)
        assert np.array_equal(table.cpu().numpy(), want["table"]) and int(plan.cursor[2]) == lacking
        out = lib.qk_norm_rope(q, k, v, plan.slots, plan.positions, None, kc, vc)
        o = lib.window_attention(out, kc, vc, table, plan.starts, plan.totals, window=window, sinks=sinks)
        at = 0
        for n in range(2):
            if new[n] < 0:
                kept[n] = [torch.zeros(0, Hkv, d, dtype=torch.float64)] * 2
                continue
            mine = slice(at, at + stored[n])
            before = len(kept[n][0])
            kept[n] = [torch.cat((a, b[mine].double().cpu())) for a, b in zip(kept[n], (k, v))]
            if counts[n]:
                # rows without a place of their own see what was stored before them
                total = before + counts[n]
                there = np.full((1, total), -1)
                there[0, :len(kept[n][0])] = np.arange(len(kept[n][0]))
                exact, absolute, _, _ = ref.attention(
                    q[at:at + counts[n]].double().cpu().numpy(), *(x.numpy()[:, None] for x in kept[n]),
                    there, [0, counts[n]], [total], window, sinks)
                got = o[at:at + counts[n]].double().cpu().numpy()
                tol = 2.0 ** -8 * np.abs(exact) + (2.0 ** -8 + 1e-5) * absolute
                assert (np.abs(got - exact) <= tol).all(), (step, n, np.abs(got - exact).max())
            at += counts[n]
        lengths, held, cursor = plan.totals, plan.pages, plan.cursor
