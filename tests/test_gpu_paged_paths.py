"""Ways through the paged cache's attention that shapes of ordinary tests do not take: loads past the caches, parts of many heads, of
per-head tables and of many sequences, and the order of row tiles of the 128-row kernel."""
import numpy as np
import pytest
import torch

from paged_util import Cache, check
from paper_2512_13368_amd import binding as B
from test_gpu_paged import TYPES, run_decode, run_prompt

pytestmark = pytest.mark.gpu


def widen(c, pages):
    """Page tables for more positions than any sequence has: what the host's choices go by.  Their entries are nobody's."""
    c.table = np.concatenate([c.table, np.full((*c.table.shape[:2], pages - c.table.shape[2]), -1, np.int32)], 2)
    c.p.max_pages, c.cap = pages, pages * c.page
    return c


def past_the_caches(c):
    return c.H // c.G <= 16 and len(c.kv_len) * c.cap * c.G * c.d * 2 * (4 if c.dtype == "fp32" else 2) > 256e6


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("split", [False, True])
def test_decode_past_the_caches(dtype, d, page, split):
    # (unsplit: as many workgroups as there are wavefronts wanted)
    S, G = (3, 2) if split else (72, 8)
    kv = ([1, 0, 700, 33, 300, 64] * 12)[:S]
    kv[2] = 1500
    pages = 1
    c = Cache(kv, 2 * G, G, d, page, dtype, seed=d + page)
    while pages * page * S * G * d * 2 * (4 if dtype == "fp32" else 2) <= 256e6 or pages < c.table.shape[2]:
        pages *= 2
    widen(c, pages)
    assert past_the_caches(c) and (B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0) == split
    c.table[2, 0, 1] = -1
    Q, O, lse = run_decode(c, strided=True)
    check(O, lse, *c.want_decode(Q), dtype)
    _, O2, lse2 = run_decode(c, Q=Q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2), "two calls on the same inputs differ"


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("H,G", [(17, 1), (40, 1), (66, 2)])
@pytest.mark.parametrize("window", [0, 1000])
def test_decode_parts_of_more_than_sixteen_heads_a_group(dtype, d, H, G, window):
    c = widen(Cache([900, 0, 1, 2100], H, G, d, 16, dtype, seed=H + d, window=window), 4096)
    assert (B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0) == (window == 0 or d >= 64 and dtype == "fp32")
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("H,G", [(6, 3), (20, 1)])
def test_decode_parts_of_tables_per_head(dtype, d, H, G):
    c = widen(Cache([900, 0, 33, 2100], H, G, d, 32, dtype, seed=H + d, per_head=True), 2048)
    assert B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0
    c.table[0, G - 1, 2], c.table[3, 0, 0] = -1, c.p.n_pages
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("bf16", 32), ("fp32", 8), ("bf16", 64), ("fp32", 128)])
@pytest.mark.parametrize("S", [63, 64, 65, 100, 127, 128])
def test_decode_parts_of_many_sequences(dtype, d, S):
    kv = [int(x) for x in np.random.default_rng(S).integers(0, 1500, S)]
    kv[3], kv[S - 1], kv[S // 2] = 0, 4000, 0
    c = Cache(kv, 2, 1, d, 32, dtype, seed=S)
    assert B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("S", [7, 8, 40, 63, 64, 65, 130, 200, 256, 257])
def test_row_tiles_of_the_128_row_kernel(d, S):
    # more than 256 tiles of 16 rows, walks of less than 8 tiles of keys, and more than 64 rows a sequence: 128 rows a workgroup, whose
    # tiles are taken by their place from 8 sequences on, up to 256
    rng = np.random.default_rng(S)
    new = [int(x) for x in rng.integers(*((201, 205) if S < 20 else (0, 5600 // S)), S)]
    new[S // 2], new[0], new[-1] = 0, min(200, 9000 // S), 1
    short = 0 if S < 20 else 64 * S // 4 + 60 - sum(new)
    while short > 0:  # (rows enough, whatever was drawn)
        i = int(rng.integers(1, S - 1))
        if i != S // 2:
            more = min(short, 30)
            new[i], short = new[i] + more, short - more
    past = [int(x) for x in rng.integers(0, 20, S)]
    c = Cache([a + b for a, b in zip(new, past)], 4, 1, d, 16, "bf16", new=new, seed=S)
    rows, tiles = 4 * c.T, -(-c.cap // 32)
    few = rows // 16 + S
    assert few > 256 and (tiles < 8 or few > 640) and (rows > 64 * S or tiles > 4), (few, tiles, rows)
    assert B.paged_workspace_bytes(c.p, B.WS_PROMPT) == 0
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), "bf16")
