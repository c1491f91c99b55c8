"""A server's loop over a cache in 4 bits that stays within a budget: prompts come in, blocks of tokens are drafted and
checked, and of every request that has grown too long each head keeps the keys that attention has used most.

One attention layer with random weights stands in for the model; how many drafted tokens the target
accepts is drawn at random. Everything else is what a serving program does each step, without a
host synchronisation:

  page_plan          where the step's tokens go
  qk_norm_rope4      queries and keys normed and rotated, keys and values into the cache in 4 bits
  window_attention4  the block against its request's keys, and each row's log of its sum of exponentials
  key_weights        how much of its attention every key has got so far, from the tokens that were accepted
  evict              requests past their limit cut to the budget, their last pages back to the queue
  topk, score_walk   the block's logits to the next draft

Run: python examples/long_context_serving.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_20530_amd as L  # noqa: E402


def rotation_table(positions: int, rot: int, device="cuda") -> torch.Tensor:
    """[positions, rot] fp32: rot / 2 cosines, then as many sines."""
    rate = 10000.0 ** (-torch.arange(rot // 2, device=device, dtype=torch.float64) / (rot // 2))
    angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * rate
    return torch.cat((angle.cos(), angle.sin()), 1).float()


class BudgetLayer:
    """One attention layer over a 4-bit cache for N requests of at most `limit` tokens plus one step's."""

    def __init__(self, N, hidden, heads, kv_heads, d, *, pages, page_size, longest, positions, budget, limit, sinks=4,
                 recent=32, decay=0.98, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.N, self.heads, self.kv, self.d = N, heads, kv_heads, d
        self.page_size, self.longest, self.decay = page_size, longest, decay
        self.bounds = dict(budget=budget, limit=limit, sinks=sinks, recent=recent)
        self.w_qkv = (r(hidden, (heads + 2 * kv_heads) * d) / hidden ** 0.5).to(dtype)
        self.w_out = (r(heads * d, hidden) / (heads * d) ** 0.5).to(dtype)
        self.q_weight, self.k_weight = 1 + 0.1 * r(d), 1 + 0.1 * r(d)
        self.cos_sin = rotation_table(positions, d)
        self.cache = L.cache4(pages, page_size, kv_heads, d)
        self.weights = torch.zeros(pages, kv_heads, page_size, device="cuda")
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((N, -(-longest // page_size)), -1, **i32)
        self.lengths, self.pages = torch.zeros(N, **i32), torch.zeros(N, 2, **i32)
        self.gone = torch.zeros(N, **i32)  # tokens that a request has lost: its positions go on behind them
        self.queue = torch.arange(pages, **i32)
        self.cursor = torch.tensor([0, pages, 0], device="cuda")

    def qkv(self, x):
        y = (x @ self.w_qkv).view(x.shape[0], self.heads + 2 * self.kv, self.d)
        return y.split((self.heads, self.kv, self.kv), 1)

    def step(self, x, incoming, tokens, most, weigh=True):
        """x [tokens, hidden], request by request; incoming [N] int32 on the device (negative: the
        request ends). tokens and most (of one request) are what the host knows. Without `weigh` the keys' weights wait
        for a call of weigh(), when it is known which tokens stay. -> [tokens, hidden]"""
        plan = L.page_plan(self.lengths, incoming, self.pages, self.table, self.queue, self.cursor,
                           page_size=self.page_size, tokens=tokens)
        self.pages, self.cursor, self.lengths = plan.pages, plan.cursor, plan.totals
        self.gone = torch.where(incoming < 0, 0, self.gone)
        if tokens == 0:
            return x
        row = torch.arange(tokens, dtype=torch.int32, device="cuda")
        request = torch.searchsorted(plan.starts[1:], row, right=True).clamp(max=self.N - 1)
        positions = torch.where(plan.positions < 0, -1, plan.positions + self.gone[request])
        q, k, v = self.qkv(x)
        q = L.qk_norm_rope4(q, k, v, plan.slots, positions, self.cos_sin, self.cache, q_weight=self.q_weight,
                            k_weight=self.k_weight)
        bounds = dict(max_tokens=most, max_length=self.longest)
        lse = torch.empty(tokens, self.heads, device="cuda")
        o = L.window_attention4(q, self.cache, self.table, plan.starts, plan.totals, lse=lse, **bounds)
        self.open = (q, lse, plan, row - plan.starts[request], request, bounds)
        if weigh:
            self.weigh()
        return o.flatten(1) @ self.w_out

    def weigh(self, accepted=None):
        """Adds what the last step's queries gave to every key; with `accepted` [N] of each request's first tokens alone
        (a row whose logarithm is -inf adds nothing). Before the lengths change."""
        q, lse, plan, token, request, bounds = self.open
        if accepted is not None:
            lse = lse.masked_fill((token >= accepted[request])[:, None], -torch.inf)
        L.key_weights(q, lse, self.cache, self.table, plan.starts, plan.totals, self.weights, decay=self.decay, **bounds)

    def cut(self):
        """Requests past their limit keep their budget."""
        e = L.evict(self.cache, self.weights, self.table, self.lengths, self.pages, self.queue, self.cursor,
                    max_length=self.longest, **self.bounds)
        self.lengths, self.pages, self.cursor, self.gone = e.totals, e.pages, e.cursor, self.gone + e.evicted

    def keep(self, lengths):
        """The requests' lengths after some of their last tokens were rejected."""
        self.lengths = lengths.to(torch.int32)


def serve(steps=12, N=8, B=16, K=8, V=32000, hidden=256, prompt=300, budget=128, limit=192, seed=0):
    """-> the drafts [steps, N, B] and the layer, after `steps` blocks of N requests."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    dt = torch.bfloat16
    layer = BudgetLayer(N, hidden, 8, 2, 64, pages=N * 24, page_size=16, longest=384, positions=prompt + B * (steps + 1),
                        budget=budget, limit=limit, seed=seed)
    E = (torch.randn(V, hidden, generator=g, device="cuda") * 0.02).to(dt)
    W = [torch.randn(hidden, hidden, generator=g, device="cuda") / hidden ** 0.5 for _ in range(2)]
    packed = L.pack_weights(*W)
    embed = lambda ids: E[ids.long().flatten()] * 16  # noqa: E731
    given = [prompt - 7 * n for n in range(N)]
    layer.step(embed(torch.randint(0, V, (sum(given),), generator=g, device="cuda")),
               torch.tensor(given, dtype=torch.int32, device="cuda"), sum(given), max(given))
    layer.cut()
    draft = torch.randint(0, V, (N, B), generator=g, device="cuda", dtype=torch.int32)
    block = torch.full((N,), B, dtype=torch.int32, device="cuda")
    drafts = []
    for s in range(steps):
        y = layer.step(embed(draft), block, N * B, B, weigh=False)
        logits = (y @ E.T).view(N, B, V)
        ids, logp = L.topk(logits, K)
        draft, _, _ = L.score_walk(ids, logp, E, packed)
        drafts.append(draft)
        accepted = torch.randint(1, B + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
        layer.weigh(accepted)  # what rejected tokens looked at counts for nothing
        # from the step's totals: a request whose pages ran out is shorter than its last one's says
        layer.keep(layer.lengths - (B - accepted))
        layer.cut()
        if s % 3 == 2:  # a request ends; the next block begins a new one in its place
            ends = torch.where(torch.arange(N, device="cuda") == s % N, -1, 0).to(torch.int32)
            layer.step(torch.empty(0, hidden, dtype=dt, device="cuda"), ends, 0, 0)
    return torch.stack(drafts), layer


def main():
    drafts, layer = serve()
    free = int(layer.cursor[1] - layer.cursor[0])
    print(f"lengths {layer.lengths.tolist()}, lost {layer.gone.tolist()}, {free} pages free, "
          f"lacking {int(layer.cursor[2])}, first draft {drafts[0, 0].tolist()}")


if __name__ == "__main__":
    main()
