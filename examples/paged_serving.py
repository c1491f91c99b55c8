"""A server's loop around the draft path over a paged cache: prompts come in, blocks of tokens are
drafted and checked, rejected tokens are rolled back, requests end and new ones take their place.

One attention layer with random weights stands in for the model; how many drafted tokens the target
accepts is drawn at random. Everything else is what a serving program does each step, without a
host synchronisation:

  page_plan          where the step's tokens go, and pages that the window left behind come back
  qk_norm_rope       queries and keys normed and rotated, keys and values into the cache
  window_attention   the block against its request's window (or prefix_attention, where all requests
                     begin with the same system prompt)
  topk, score_walk   the block's logits to the next draft

Run: python examples/paged_serving.py
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


class PagedLayer:
    """One attention layer over a paged cache for N requests at a time."""

    def __init__(self, N, hidden, heads, kv_heads, d, *, pages, page_size, longest, window=0, sinks=0,
                 shared=0, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.N, self.heads, self.kv, self.d = N, heads, kv_heads, d
        self.page_size, self.window, self.sinks, self.longest = page_size, window, sinks, longest
        self.w_qkv = (r(hidden, (heads + 2 * kv_heads) * d) / hidden ** 0.5).to(dtype)
        self.w_out = (r(heads * d, hidden) / (heads * d) ** 0.5).to(dtype)
        self.q_weight, self.k_weight = 1 + 0.1 * r(d), 1 + 0.1 * r(d)
        self.cos_sin = rotation_table(longest + shared, d)
        self.k_cache = torch.zeros(pages, page_size, kv_heads, d, dtype=dtype, device="cuda")
        self.v_cache = torch.zeros_like(self.k_cache)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.shared, held = shared, -(-shared // page_size)  # the first pages hold the system prompt
        self.shared_table = torch.arange(held, **i32)
        self.table = torch.full((N, -(-longest // page_size)), -1, **i32)
        self.lengths, self.pages = torch.zeros(N, **i32), torch.zeros(N, 2, **i32)
        self.queue = torch.roll(torch.arange(pages, **i32), -held)  # every other page is free
        self.cursor = torch.tensor([0, pages - held, 0], device="cuda")
        self.spare = None  # the plan that the next step may overwrite
        self.workspaces = {}

    def qkv(self, x):
        y = (x @ self.w_qkv).view(x.shape[0], self.heads + 2 * self.kv, self.d)
        return y.split((self.heads, self.kv, self.kv), 1)

    def write_shared(self, x):
        """The system prompt's keys and values, once."""
        at = torch.arange(self.shared, dtype=torch.int32, device="cuda")
        q, k, v = self.qkv(x)
        L.qk_norm_rope(q, k, v, at, at, self.cos_sin, self.k_cache, self.v_cache,
                       q_weight=self.q_weight, k_weight=self.k_weight)

    def step(self, x, incoming, tokens, most):
        """x [tokens, hidden], request by request; incoming [N] int32 on the device (negative: the
        request ends). tokens and most (of one request) are what the host knows. -> [tokens, hidden]"""
        out = self.spare if self.spare is not None and self.spare.slots.numel() == tokens else None
        plan = L.page_plan(self.lengths, incoming, self.pages, self.table, self.queue, self.cursor,
                           page_size=self.page_size, tokens=tokens, window=self.window, sinks=self.sinks,
                           out=out)
        self.spare = getattr(self, "plan", None)
        self.plan, self.pages, self.cursor = plan, plan.pages, plan.cursor
        q, k, v = self.qkv(x)
        q = L.qk_norm_rope(q, k, v, plan.slots, plan.positions, self.cos_sin[self.shared:], self.k_cache,
                           self.v_cache, q_weight=self.q_weight, k_weight=self.k_weight)
        bounds = dict(max_tokens=most, max_length=self.longest)
        kind = (tokens, most)
        if self.shared:
            if kind not in self.workspaces:
                self.workspaces[kind] = L.prefix_attention_workspace(q, self.k_cache, self.table,
                                                                     self.shared, **bounds)
            o = L.prefix_attention(q, self.k_cache, self.v_cache, self.shared_table, self.shared,
                                   self.table, plan.starts, plan.totals, workspace=self.workspaces[kind],
                                   **bounds)
        else:
            mask = dict(window=self.window, sinks=self.sinks)
            if kind not in self.workspaces:
                self.workspaces[kind] = L.window_attention_workspace(q, self.k_cache, self.table, **mask,
                                                                     **bounds)
            o = L.window_attention(q, self.k_cache, self.v_cache, self.table, plan.starts, plan.totals,
                                   workspace=self.workspaces[kind], **mask, **bounds)
        self.lengths = plan.totals
        return o.flatten(1) @ self.w_out

    def keep(self, lengths):
        """The requests' lengths after some of their last tokens were rejected."""
        self.lengths = lengths.to(torch.int32)


def serve(steps=6, N=8, B=16, K=8, V=32000, hidden=256, prompt=200, window=128, sinks=4, shared=0, seed=0):
    """-> the drafts [steps, N, B] and the layer, after `steps` blocks of N requests."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    dt = torch.bfloat16
    layer = PagedLayer(N, hidden, 8, 2, 64, pages=N * 64 + 64, page_size=16, longest=1024,
                       window=0 if shared else window, sinks=0 if shared else sinks, shared=shared, seed=seed)
    E = (torch.randn(V, hidden, generator=g, device="cuda") * 0.02).to(dt)
    W = [torch.randn(hidden, hidden, generator=g, device="cuda") / hidden ** 0.5 for _ in range(2)]
    packed = L.pack_weights(*W)
    embed = lambda ids: E[ids.long().flatten()] * 16  # noqa: E731
    if shared:
        layer.write_shared(embed(torch.randint(0, V, (shared,), generator=g, device="cuda")))
    # prompts of different lengths, all in one step
    given = [prompt - 7 * n for n in range(N)]
    layer.step(embed(torch.randint(0, V, (sum(given),), generator=g, device="cuda")),
               torch.tensor(given, dtype=torch.int32, device="cuda"), sum(given), max(given))
    draft = torch.randint(0, V, (N, B), generator=g, device="cuda", dtype=torch.int32)
    block = torch.full((N,), B, dtype=torch.int32, device="cuda")
    drafts = []
    for s in range(steps):
        y = layer.step(embed(draft), block, N * B, B)
        logits = (y @ E.T).view(N, B, V)
        ids, logp = L.topk(logits, K)
        draft, _, _ = L.score_walk(ids, logp, E, packed)
        drafts.append(draft)
        accepted = torch.randint(1, B + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
        # from the step's totals: a request whose pages ran out is shorter than its last one's says
        layer.keep(layer.lengths - (B - accepted))
        if s % 3 == 2:  # a request ends; the next block begins a new one in its place
            ends = torch.where(torch.arange(N, device="cuda") == s % N, -1, 0).to(torch.int32)
            layer.step(torch.empty(0, hidden, dtype=dt, device="cuda"), ends, 0, 0)
    return torch.stack(drafts), layer


def main():
    for shared in (0, 300):
        drafts, layer = serve(shared=shared)
        free = int(layer.cursor[1] - layer.cursor[0])
        print(f"shared prompt of {shared}: lengths {layer.lengths.tolist()}, {free} pages free, "
              f"lacking {int(layer.cursor[2])}, first draft {drafts[0, 0].tolist()}")


if __name__ == "__main__":
    main()
