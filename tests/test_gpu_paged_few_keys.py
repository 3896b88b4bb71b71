"""Rows that see few keys inside large bf16 prompts: their probabilities are large, and the bound on an output goes by the root mean square
of all outputs, most of which are averages over many keys."""
import numpy as np
import pytest
import torch

from paged_util import Cache, check
from paper_2512_13368_amd import binding as B
from test_gpu_paged import CROWD, TYPES, run_prompt
from test_gpu_paged_paths import widen
from test_gpu_paged_probabilities import check_fine, coarse, coarse_keys

pytestmark = pytest.mark.gpu

DIMS = [8, 16, 32, 64, 128]


def few(c, s, i):
    """Whether new token i of sequence s sees fewer than 32 keys."""
    pos = c.kv_len[s] - c.new[s] + i
    lo = max(pos - c.window + 1, 0) if c.window else 0
    return 0 <= pos and len(c.keys(s, 0, lo, min(pos + 1, c.kv_len[s]))[0]) < 32


def rows_of_few_keys(c):
    rows = [(int(c.cu[s]) + i, s, c.kv_len[s] - c.new[s] + i) for s in range(len(c.new)) for i in range(c.new[s]) if few(c, s, i)]
    assert len(rows) > 20
    return rows


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("H,G", [(2, 1), (6, 2), (1, 1)])
@pytest.mark.parametrize("window", [0, 20])
def test_sequences_begin_with_few_keys(d, H, G, window):
    new, kv = [150, 1, 40, 33, 9], [150, 1, 43, 200, 31]
    c = Cache(kv + [0] * CROWD, H, G, d, 16, "bf16", new=new + [0] * CROWD, seed=d, window=window, scale=0.5 * d**-0.5)
    coarse_keys(c)
    Q, O, _ = run_prompt(c, Q=coarse(c, c.T, H, d))
    check_fine(c, O, Q, rows_of_few_keys(c))


@pytest.mark.parametrize("d", DIMS)
def test_so_do_walks_that_are_split(d):
    c = widen(Cache([150, 1, 43, 400], 4, 2, d, 16, "bf16", new=[150, 1, 40, 390], seed=d, scale=0.5 * d**-0.5), 40000)
    assert B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0
    coarse_keys(c)
    Q, O, _ = run_prompt(c, Q=coarse(c, c.T, 4, d))
    check_fine(c, O, Q, rows_of_few_keys(c))


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("page", [8, 16, 32])
def test_missing_pages_leave_few_keys(d, page):
    # all but a page or two out of range, among them the first, one inside, and the last; 32 positions or more before every token
    n = 200
    c = Cache([n, n, n] + [0] * CROWD, 2, 1, d, page, "bf16", new=[100, 90, 50] + [0] * CROWD, seed=d, scale=0.5 * d**-0.5)
    coarse_keys(c)
    keep = [{0, 96 // page}, {64 // page}, {(n - 1) // page}]
    for s, pages in enumerate(keep):
        for i in range(c.table.shape[2]):
            if i not in pages:
                c.table[s, 0, i] = -1 if i % 2 else c.p.n_pages
    Q, O, _ = run_prompt(c, Q=coarse(c, c.T, 2, d))
    check_fine(c, O, Q, rows_of_few_keys(c))


@pytest.mark.parametrize("d", DIMS)
def test_tokens_beyond_the_capacity_see_few_keys(d):
    c = Cache([170] + [0] * CROWD, 2, 1, d, 16, "bf16", new=[150] + [0] * CROWD, seed=d, scale=0.5 * d**-0.5, window=70, max_len=90)
    coarse_keys(c)
    Q, O, _ = run_prompt(c, Q=coarse(c, c.T, 2, d))
    check_fine(c, O, Q, rows_of_few_keys(c))


@pytest.mark.parametrize("d", DIMS)
def test_a_long_prompt_keeps_the_bound_from_its_first_token_on(d):
    c = Cache([2048, 7], 4, 2, d, 32, "bf16", new=[2048, 7], seed=d)
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), "bf16")


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("form", ["few rows", "many rows", "split"])
def test_entries_behind_the_window_change_nothing(dtype, d, form):
    # a cache that gives pages back once the window has passed them: not a bit of the results depends on their entries
    kv, new = [2000, 900, 130], {"few rows": [3, 1, 2], "many rows": [150, 40, 130], "split": [150, 40, 130]}[form]
    crowd = CROWD if form == "many rows" else 0
    c = Cache(kv + [0] * crowd, 4, 2, d, 16, dtype, new=new + [0] * crowd, window=100 if form != "split" else 1300, seed=d)
    assert (B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0) == (form == "split")
    Q, O, lse = run_prompt(c)
    for s, (n, m) in enumerate(zip(kv, new)):
        c.table[s, 0, :max(0, n - m - c.window + 1) // 16] = -1
    assert (c.table[0, 0, :20] == -1).all()
    _, O2, lse2 = run_prompt(c, Q=Q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    check(O, lse, *c.want_prompt(Q), dtype)
