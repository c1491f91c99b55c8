"""Page plans with fewer rows than new tokens: the tokens past the last row are not taken, and starts and totals
say so together, so that the queries that there are keep their positions and see no key that has no row."""
import numpy as np
import pytest
import torch

import oracle.paged as ref

LENGTHS, INCOMING = [5, 0, 9, 30, 2], [4, 6, 3, -1, 7]


def test_rows_by_hand():
    table = np.full((5, 8), -1, np.int32)
    pages = [(2, 0), (0, 0), (3, 0), (8, 0), (1, 0)]
    got = ref.page_plan(LENGTHS, INCOMING, pages, table, np.arange(20, dtype=np.int32), [0, 20, 0], 4, 8)
    assert got["starts"].tolist() == [0, 4, 8, 8, 8, 8]
    assert got["totals"].tolist() == [9, 4, 9, 0, 2]
    assert got["positions"].tolist() == [5, 6, 7, 8, 0, 1, 2, 3]


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [0, 1, 4, 8, 13, 19, 20, 25])
def test_rows(lib, tokens):
    P, M = 4, 8
    pages = [(-(-n // P), 0) for n in LENGTHS]
    rng = np.random.default_rng(tokens)
    order = rng.permutation(40).astype(np.int32)
    table, at = np.full((5, M), -1, np.int32), 0
    for n, (end, _) in enumerate(pages):
        table[n, :end] = order[at:at + end]
        at += end
    host = dict(lengths=np.array(LENGTHS, np.int32), incoming=np.array(INCOMING, np.int32),
                pages=np.array(pages, np.int32), table=table, queue=np.roll(order, -at),
                cursor=np.array([0, 40 - at, 0], np.int64))
    dev = {k: torch.from_numpy(v).cuda() for k, v in host.items()}
    plan = lib.page_plan(**dev, page_size=P, tokens=tokens)
    want = ref.page_plan(**host, page_size=P, tokens=tokens)
    got = {k: getattr(plan, k) for k in plan._fields} | {k: dev[k] for k in ("table", "queue")}
    for k, v in want.items():
        assert np.array_equal(got[k].cpu().numpy(), v), (k, got[k], v)
