"""The paged cache's attention where logits are finite and far from 0: the key with the largest logit keeps a weight of 1 of its own
size, whatever the rounding of the softmax's reference is in units of the exponent (2^13 at logits of 1e11)."""
import numpy as np
import pytest
import torch

from paged_util import DTYPES, Cache, check
from paper_2512_13368_amd import binding as B
from test_gpu_paged import CROWD, TYPES, run_decode, run_prompt

pytestmark = pytest.mark.gpu

ODD = np.array([181, 179, 173, 167, 163, 157, 151, 149, 139, 137])  # of 8 bits: products with each other are exact in 16


def keys(kind, n):
    """Of each position the one channel that is not 0, exact in bf16; products with the queries' are exact in fp32."""
    j = np.arange(n)
    if kind == "equal":        # the mean of the values
        return np.full(n, 181.0 * 2.0**24)
    if kind == "equal, below 0":
        return np.full(n, -181.0 * 2.0**24)
    if kind == "steps":        # several largest ones, far above the rest
        return (128.0 + 13 * j % 97) * 2.0**24
    if kind == "growing":      # from ordinary logits to the largest
        return ODD[j % 10] * 2.0 ** (np.minimum(j // 7, 30) - 6)
    return ODD[j % 10] * 2.0 ** (24 - np.minimum(j // 7, 30))


KINDS = ["equal", "equal, below 0", "steps", "growing", "falling"]


def fill(c, kind):
    for s, n in enumerate(c.kv_len):
        if n:
            a = torch.from_numpy(keys(kind, n)).to(DTYPES[c.dtype])
            for g in range(c.G):
                ids, j = torch.from_numpy(c.table[s, 0].astype(np.int64))[np.arange(n) // c.page], torch.arange(n) % c.page
                c.K_cache[ids, g, j] = 0
                c.K_cache[ids, g, j, 0] = a


def queries(c, rows):
    """Large, but every third row sees ordinary logits, or none but 0."""
    Q = torch.zeros(rows, c.H, c.d, dtype=DTYPES[c.dtype])
    for h in range(c.H):
        Q[:, h, 0] = torch.from_numpy(ODD[(np.arange(rows) + h) % 10] * 1.0).to(Q.dtype)
    Q[2::3] = 0
    return Q


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("split", [False, True])
def test_decode(dtype, d, kind, split):
    c = Cache([1, 300, 64, 0, 31], 4, 2, d, 16, dtype, seed=d, max_pages=4096 if split else None)
    assert (B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0) == split
    fill(c, kind)
    Q, O, lse = run_decode(c, Q=queries(c, 5))
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", ["few rows", "many rows", "many rows, split"])
def test_prompt(dtype, d, kind, form):
    kv, new = [1, 300, 64, 31], [1, 120, 64, 5]
    if form == "few rows":
        kv, new = [1, 300, 64, 31], [1, 9, 2, 5]
    crowd = CROWD if form == "many rows" else 0
    c = Cache(kv + [0] * crowd, 8, 2, d, 16, dtype, new=new + [0] * crowd, seed=d, max_pages=40000 if form == "many rows, split" else None)
    if form == "many rows, split":
        assert B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0
    fill(c, kind)
    Q, O, lse = run_prompt(c, Q=queries(c, c.T))
    check(O, lse, *c.want_prompt(Q), dtype)
