"""Drafted trees, forked pages and beams for tests: their definitions in 64 bits on the CPU."""
import numpy as np
import torch

from paged_util import Cache


def tree_masks(parents):
    """Masks of one sequence's drafted tokens from their parents (-1: the history): a token sees itself and its ancestors."""
    masks = []
    for i, up in enumerate(parents):
        masks.append((1 << i if i < 64 else 0) | (masks[up] if up >= 0 else 0))
    return masks


def signed(mask):
    return mask - (1 << 64) if mask >= 1 << 63 else mask


class TreeCache(Cache):
    """A cache whose `new` tokens are drafted trees, with random parents unless masks are given."""

    def __init__(self, kv_len, *args, masks=None, seed=0, **kw):
        super().__init__(kv_len, *args, seed=seed, **kw)
        rng = np.random.default_rng(seed + 1000)
        if masks is None:
            masks = [tree_masks([int(rng.integers(-1, i)) if i else -1 for i in range(n)]) for n in self.new]
        self.masks = [m for one in masks for m in one]

    def mask(self):
        rows = self.masks + [0] * (self.T - len(self.masks))
        return torch.tensor([signed(m) for m in rows], dtype=torch.int64).cuda()

    def sees(self, s, i):
        """(position, [slots of the drafted tokens seen]) of token i of a sequence."""
        n, m = self.new[s], self.masks[int(self.cu[s]) + i]
        past = max(self.kv_len[s], 0) - n
        named = [k for k in range(min(n, 64)) if m >> k & 1]
        return past + len([k for k in named if k != i]), [past + k for k in named if 0 <= past + k < self.cap]

    def attend_tree(self, q, s, i, h):
        n = self.new[s]
        past = max(self.kv_len[s], 0) - n
        pos, drafted = self.sees(s, i)
        g = h // (self.H // self.G)
        lo = max(max(past, 0) + (pos - past) - self.window + 1, 0) if self.window else 0
        parts = [self.keys(s, g, lo, past)] + [self.keys(s, g, j, j + 1) for j in drafted]
        k, v = torch.cat([p[1] for p in parts]), torch.cat([p[2] for p in parts])
        if len(k) == 0:
            return torch.zeros(self.d, dtype=torch.float64), float("-inf")
        x = (k @ q.double()) * self.scale
        lse = torch.logsumexp(x, 0)
        return torch.exp(x - lse) @ v, float(lse)

    def want_tree(self, Q):
        O, lse = torch.zeros(Q.shape, dtype=torch.float64), torch.zeros(Q.shape[:2], dtype=torch.float64)
        for s in range(len(self.kv_len)):
            for i in range(self.new[s]):
                t = int(self.cu[s]) + i
                for h in range(self.H):
                    O[t, h], lse[t, h] = self.attend_tree(Q[t, h], s, i, h)
        return O, lse


def want_fork(table, kv_len, refs, parent, page, cap, grow):
    """(new_table, new_len, new_refs, copies, missing) by the definition, on lists of whole numbers."""
    S, width, n_pages = len(table), len(table[0]), len(refs)

    def real(p):
        return 0 <= p < n_pages

    before, refs = list(refs), list(refs)
    for row in table:
        for p in row:
            if real(p):
                refs[p] -= 1
    seen, rows, lens, copies, wanted = set(), [], [], [], []
    for n, q in enumerate(parent):
        row, copies_n, length = [-1] * width, [-1, -1, 0], 0
        if 0 <= q < S:
            length = min(max(kv_len[q], 0), cap)
            full, part = divmod(length, page)
            need = -(-min(length + grow, cap) // page)
            eldest = q not in seen
            seen.add(q)
            for i in range(need):
                p = table[q][i] if real(table[q][i]) else -1
                if i < full or (eldest and p >= 0 and before[p] == 1):
                    row[i] = p
                    if p >= 0:
                        refs[p] += 1
                    continue
                wanted.append((n, i))
                if i == full and part and p >= 0:
                    copies_n = [p, -1, part]
        rows.append(row)
        lens.append(length)
        copies.append(copies_n)
    kept = {c[0] for c in copies if c[0] >= 0}
    spare = iter([p for p in range(n_pages) if refs[p] == 0 and p not in kept])
    missing = 0
    for n, i in wanted:
        p = next(spare, -1)
        if p < 0:
            missing += 1
        else:
            refs[p] += 1
            rows[n][i] = p
        if copies[n][0] >= 0 and i == lens[n] // page:
            copies[n] = [copies[n][0], p, copies[n][2]] if p >= 0 else [-1, -1, 0]
    return rows, lens, refs, copies, [missing]


def want_beam(logits, score, K, ended=None, eos=-1):
    """(parent, token, score, ended) by the definition: every candidate in its place in the order."""
    B, W = score.shape
    x = logits.double().numpy().reshape(B, W, -1)
    out = np.full((B, K), -1, np.int32), np.full((B, K), -1, np.int32), np.full((B, K), -np.inf), np.zeros((B, K), bool)
    for b in range(B):
        rows = []
        for w in range(W):
            c = float(score[b, w])
            if ended is not None and bool(ended[b, w]):
                rows.append((np.array([c]), np.zeros(1), np.array([eos]), np.full(1, w)))
                continue
            r = np.where(np.isnan(x[b, w]), -np.inf, x[b, w])
            m = r.max()
            if not np.isfinite(m) or np.isnan(c):
                continue
            to = c + (r - (m + np.log(np.exp(r - m).sum())))
            rows.append((to, r, np.arange(r.size), np.full(r.size, w)))
        if not rows:
            continue
        to, r, v, w = (np.concatenate(c) for c in zip(*rows))
        ok = ~np.isnan(to) & (to > -np.inf)
        to, r, v, w = to[ok], r[ok], v[ok], w[ok]
        at = np.lexsort((v, -r, w, -to))[:K]
        out[0][b, :len(at)], out[1][b, :len(at)], out[2][b, :len(at)] = b * W + w[at], v[at], to[at]
        out[3][b, :len(at)] = (v[at] == eos) | (ended is not None and np.asarray(ended[b])[w[at]].astype(bool))
    return out
