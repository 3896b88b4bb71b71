#!/usr/bin/env python3
"""Serving from a paged key/value cache: histories are taken in once, then grow by an item at a time.

One attention layer of a sequential recommender with random weights.  Users' histories of different lengths come as one packed
batch (kv_append, attn_prompt); then every user gets new items, one a step (kv_append, attn_decode).  Beside full attention a step
shows the two branches of Blossom attention for a single new token: the long-term branch reads the pages whose mean key scores best
for each key/value head (a page table per head), the short-term branch a window, and a gate blends them.  (The pages are chosen in
plain torch from the whole cache: it shows what the calls take, not how fast a selection can be.)

    python examples/serve_paged.py [--users 32] [--history 1000] [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2512_13368_amd import binding as B  # noqa: E402
from paper_2512_13368_amd.inputs import rope_tables  # noqa: E402

HEADS, GROUPS, DIM, PAGE, TOPK, WINDOW = 8, 2, 64, 32, 8, 64
WIDTH = HEADS * DIM


class Layer:
    """The layer's weights, and its cache: pages for every user, handed out as histories grow."""

    def __init__(self, users: int, capacity: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.users, self.width = users, -(-capacity // PAGE)
        n_pages = users * self.width
        self.W_qkv = (normal(WIDTH, (HEADS + 2 * GROUPS) * DIM) * WIDTH ** -0.5).bfloat16()
        self.gate_w = normal(HEADS, 2 * DIM) * 0.02
        self.K_cache = torch.zeros(n_pages, GROUPS, PAGE, DIM, dtype=torch.bfloat16, device="cuda")
        self.V_cache = torch.zeros_like(self.K_cache)
        self.free = torch.randperm(n_pages, generator=g, device="cuda").tolist()
        self.table = torch.full((users, self.width), -1, dtype=torch.int32)
        self.rope = tuple(torch.from_numpy(t).cuda() for t in rope_tables(self.width * PAGE, DIM))
        self.kv_len = torch.zeros(users, dtype=torch.int32)

    def params(self, tokens: int, **kw) -> B.PagedParams:
        p = dict(S=self.users, T=tokens, H=HEADS, G=GROUPS, d=DIM, page=PAGE, n_pages=self.K_cache.shape[0], max_pages=self.width, dtype=B.BF16)
        return B.PagedParams(**{**p, **kw})

    def grow(self, new: list[int]) -> tuple[torch.Tensor, torch.Tensor]:
        """Makes room for new[u] more items of user u.  Returns (cu_seqlens, kv_len) on the GPU."""
        for u, n in enumerate(new):
            have, self.kv_len[u] = -(-int(self.kv_len[u]) // PAGE), int(self.kv_len[u]) + n
            for i in range(have, -(-int(self.kv_len[u]) // PAGE)):
                self.table[u, i] = self.free.pop()
        self.table_dev = self.table.cuda()
        cu = torch.tensor([0, *new]).cumsum(0).to(torch.int32).cuda()
        return cu, self.kv_len.cuda()

    def append(self, x: torch.Tensor, cu: torch.Tensor, kv_len: torch.Tensor) -> torch.Tensor:
        """Projects packed items x [T, WIDTH], stores their keys and values, returns the rotated queries."""
        qkv = x @ self.W_qkv
        q, k, v = (t.unflatten(1, (-1, DIM)) for t in qkv.split([HEADS * DIM, GROUPS * DIM, GROUPS * DIM], 1))
        return B.kv_append(self.params(x.shape[0]), k, v, self.K_cache, self.V_cache, self.table_dev, cu, kv_len, Q=q, rope=self.rope)

    def prompt(self, x: torch.Tensor, new: list[int]) -> torch.Tensor:
        cu, kv_len = self.grow(new)
        q = self.append(x, cu, kv_len)
        return B.attn_prompt(self.params(x.shape[0]), q, self.K_cache, self.V_cache, self.table_dev, cu, kv_len)[0]

    def step(self, x: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
        """One new item for every user: (full attention, Blossom attention)."""
        cu, kv_len = self.grow([1] * self.users)
        q = self.append(x, cu, kv_len)
        full, _ = B.attn_decode(self.params(x.shape[0]), q, self.K_cache, self.V_cache, self.table_dev, kv_len)
        st, _ = B.attn_decode(self.params(x.shape[0], window=WINDOW), q, self.K_cache, self.V_cache, self.table_dev, kv_len)
        table, listed = self.select(q, kv_len)
        p = self.params(x.shape[0], max_pages=table.shape[2], table_per_head=1)
        lt, _ = B.attn_decode(p, q, self.K_cache, self.V_cache, table, listed)
        both = torch.cat([lt, st], -1).float()
        alpha = torch.sigmoid((both * self.gate_w).sum(-1, keepdim=True))
        return full, (alpha * lt.float() + (1 - alpha) * st.float()).to(full.dtype)

    def select(self, q: torch.Tensor, kv_len: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
        """Per user and key/value head the newest page and the TOPK - 1 best earlier ones, in ascending order, as a table of
        pages; and how many positions they hold (the listed pages are whole but the newest).  This shows the table's form: it takes
        every page's mean anew, which reads more than full attention does.  A program that selects for speed keeps the means of whole
        pages beside the cache."""
        pages = self.table_dev.long().clamp(min=0)
        mean = self.K_cache[pages].float().mean(3).permute(0, 2, 1, 3)                    # [users, G, pages, DIM]
        mine = q.float().view(self.users, GROUPS, HEADS // GROUPS, DIM).sum(2)
        score = torch.matmul(mean, mine[..., None])[..., 0]
        newest = ((kv_len.long() - 1) // PAGE)[:, None, None]
        at = torch.arange(self.width, device="cuda")
        score = torch.where(at < newest, score, torch.full_like(score, -torch.inf)).masked_fill(at == newest, torch.inf)
        k = min(TOPK, self.width)
        real = (newest + 1).clamp(max=k)
        best = score.topk(k, dim=2).indices
        best = torch.where(torch.arange(k, device="cuda") < real, best, torch.full_like(best, self.width)).sort(dim=2).values
        ids = torch.cat([self.table_dev, torch.full((self.users, 1), -1, dtype=torch.int32, device="cuda")], 1)
        table = ids[torch.arange(self.users, device="cuda")[:, None, None], best].contiguous()
        return table, ((real[:, 0, 0] - 1) * PAGE + (kv_len.long() - 1) % PAGE + 1).to(torch.int32)


def main(users: int = 32, history: int = 1000, steps: int = 8, seed: int = 0) -> float:
    """Runs the requests; returns how far a step's full attention is from the same item inside one long prompt."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    lengths = [max(1, history * (u + 1) // users) for u in range(users)]
    items = [torch.randn(n + steps, WIDTH, generator=g, device="cuda").bfloat16() for n in lengths]
    layer = Layer(users, history + steps, seed)
    layer.prompt(torch.cat([x[:n] for x, n in zip(items, lengths)]), lengths)
    for i in range(steps):
        full, blossom = layer.step(torch.stack([x[n + i] for x, n in zip(items, lengths)]))
    again = Layer(users, history + steps, seed)
    whole = again.prompt(torch.cat(items), [n + steps for n in lengths])
    last = torch.tensor([n + steps for n in lengths]).cumsum(0) - 1
    off = float((whole[last.cuda()].float() - full.float()).abs().max())
    print(f"{users} users, histories of {lengths[0]} to {lengths[-1]} items, {steps} steps: the last item's attention differs from that of "
          f"a prompt over everything by at most {off:.2e}; Blossom attention of it has norm {float(blossom.float().norm()):.3f}")
    return off


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--users", type=int, default=32)
    a.add_argument("--history", type=int, default=1000)
    a.add_argument("--steps", type=int, default=8)
    main(**vars(a.parse_args()))
