"""A paged key/value cache for tests, and its operators' definitions in 64 bits on the CPU, one sequence and head at a time."""
import numpy as np
import torch

from paper_2512_13368_amd import binding as B

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
JUNK = float("nan")  # what no call may read into a result: slots beyond a sequence's end, pages that nobody lists


class Cache:
    """S sequences of kv_len positions; `new` of each are the tokens a call brings (default 1).  Every row that a sequence does not
    hold is NaN, and page-table entries beyond its last page are out of range in one way or another."""

    def __init__(self, kv_len, H, G, d, page, dtype, new=None, per_head=False, seed=0, spare=2, max_pages=None, window=0, max_len=0,
                 scale=0.0, fill=True):
        rng = np.random.default_rng(seed)
        self.kv_len = [int(n) for n in kv_len]
        S = len(self.kv_len)
        self.new = [1] * S if new is None else [int(n) for n in new]
        self.H, self.G, self.d, self.page, self.dtype, self.window = H, G, d, page, dtype, window
        dt = DTYPES[dtype]
        need = [-(-max(n, 0) // page) for n in self.kv_len]
        width = max_pages or max(max(need), 1)
        heads = G if per_head else 1
        n_pages = heads * S * width + spare
        order = rng.permutation(n_pages)[:heads * S * width].reshape(S, heads, width)
        self.table = order.astype(np.int32)
        for s in range(S):
            for i in range(min(need[s], width), width):
                self.table[s, :, i] = rng.choice([-1, n_pages, 2**31 - 1, -2**31, int(order[s, 0, i])])
        self.cap = min(width * page, max_len) if max_len else width * page
        self.K_cache = torch.full((n_pages, G, page, d), JUNK, dtype=dt)
        self.V_cache = torch.full((n_pages, G, page, d), JUNK, dtype=dt)
        if fill:
            for s in range(S):
                for g in range(G):
                    n = min(max(self.kv_len[s], 0), width * page)
                    if n == 0:
                        continue
                    j = torch.arange(n)
                    ids = torch.from_numpy(order[s, g if per_head else 0].astype(np.int64))[j // page]
                    self.K_cache[ids, g, j % page] = torch.from_numpy(rng.standard_normal((n, d), dtype=np.float32)).to(dt)
                    self.V_cache[ids, g, j % page] = torch.from_numpy(rng.standard_normal((n, d), dtype=np.float32)).to(dt)
        self.T = max(1, sum(self.new))
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.rng, self.per_head = rng, per_head
        self.p = B.PagedParams(S=S, T=self.T, H=H, G=G, d=d, page=page, n_pages=n_pages, max_pages=width,
                               dtype=B.F32 if dtype == "fp32" else B.BF16, softmax_scale=scale, window=window, max_len=max_len,
                               table_per_head=int(per_head))
        self.scale = scale or d ** -0.5

    def normal(self, *shape):
        return torch.from_numpy(self.rng.standard_normal(shape, dtype=np.float32)).to(DTYPES[self.dtype])

    def dev(self):
        """(K_cache, V_cache, page_table, cu_seqlens, kv_len) on the GPU."""
        table = self.table if self.per_head else self.table[:, 0]
        return (self.K_cache.cuda(), self.V_cache.cuda(), torch.from_numpy(np.ascontiguousarray(table)).cuda(),
                torch.from_numpy(self.cu).cuda(), torch.tensor(self.kv_len, dtype=torch.int32).cuda())

    def keys(self, s, g, lo, hi):
        """Positions lo .. hi-1 of a sequence that have a page, and their K and V in 64 bits."""
        j = np.arange(max(lo, 0), min(hi, self.cap))
        ids = self.table[s, g if self.per_head else 0][j // self.page].astype(np.int64)
        ok = (ids >= 0) & (ids < self.K_cache.shape[0])
        j, ids = torch.from_numpy(j[ok]), torch.from_numpy(ids[ok])
        return j, self.K_cache[ids, g, j % self.page].double(), self.V_cache[ids, g, j % self.page].double()

    def attend(self, q, s, h, pos):
        """(o, lse) of one query in 64 bits."""
        n = self.kv_len[s]
        lo = pos - self.window + 1 if self.window else 0
        none = torch.zeros(self.d, dtype=torch.float64), float("-inf")
        if pos < 0 or min(pos + 1, n) <= max(lo, 0):
            return none
        _, k, v = self.keys(s, h // (self.H // self.G), lo, min(pos + 1, n))
        if len(k) == 0:
            return none
        x = (k @ q.double()) * self.scale
        lse = torch.logsumexp(x, 0)
        return torch.exp(x - lse) @ v, float(lse)

    def want_decode(self, Q):
        O, lse = torch.zeros(Q.shape, dtype=torch.float64), torch.zeros(Q.shape[:2], dtype=torch.float64)
        for s in range(len(self.kv_len)):
            for h in range(self.H):
                O[s, h], lse[s, h] = self.attend(Q[s, h], s, h, self.kv_len[s] - 1)
        return O, lse

    def want_prompt(self, Q):
        O, lse = torch.zeros(Q.shape, dtype=torch.float64), torch.zeros(Q.shape[:2], dtype=torch.float64)
        for s in range(len(self.kv_len)):
            for i in range(self.new[s]):
                for h in range(self.H):
                    t = self.cu[s] + i
                    O[t, h], lse[t, h] = self.attend(Q[t, h], s, h, self.kv_len[s] - self.new[s] + i)
        return O, lse


# The contract's accuracy: |x - ref| <= tol * (|ref| + rms(ref)).
TOL = {"fp32": 1e-4, "bf16": 2e-2}
# A logit is a sum of d products in fp32, each addition off by 2^-24 of the running sum at most: with unit normal channels and the
# scale 1/sqrt(d), d * 2^-24 * sqrt(d) * 2/pi is 5.5e-5 at d = 128; the log of the sum of exponentials is off by no more than its
# largest logit, and by fp32's own rounding of the result.
LSE_TOL = 6e-5


def check(O, lse, want_O, want_lse, dtype):
    got = O.double().cpu()
    assert torch.isfinite(got).all(), "outputs that are not finite"
    rms = float(want_O.pow(2).mean().sqrt())
    off = (got - want_O).abs() - TOL[dtype] * (want_O.abs() + rms)
    assert float(off.max()) <= 0, f"O off by {float(off.max()):.3g} beyond the bound at {np.unravel_index(int(off.argmax()), off.shape)}"
    got = lse.double().cpu()
    empty = torch.isinf(want_lse)
    assert torch.equal(got[empty], want_lse[empty]), "lse of rows that see nothing"
    off = (got[~empty] - want_lse[~empty]).abs() - LSE_TOL * (1 + want_lse[~empty].abs())
    assert off.numel() == 0 or float(off.max()) <= 0, f"lse off by {float(off.max()):.3g} beyond the bound"


def guarded(rows, heads, d, dtype):
    """An output tensor with marked rows behind it, and a function that says whether those are untouched."""
    whole = torch.full((rows + 4, heads, d), 7.0, dtype=DTYPES[dtype], device="cuda")
    return whole[:rows], lambda: bool((whole[rows:] == 7.0).all())
