"""Drafted trees where logits are large, grow along the keys, or are -inf: at the bounds that prompts are held to."""
import numpy as np
import pytest
import torch

from paged_util import DTYPES, check
from paper_2512_13368_amd import binding as B
from test_gpu_paged import TYPES, check_grown, growing
from test_gpu_paged_large_logits import KINDS, fill, queries
from test_gpu_tree import run_tree
from tree_util import TreeCache

pytestmark = pytest.mark.gpu


def cut(c):
    return B.paged_workspace_bytes(c.p, B.WS_TREE) > 0


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("tokens", [4, 20, 64])
@pytest.mark.parametrize("split", [False, True])
def test_logits_that_grow_along_the_keys(dtype, d, tokens, split):
    c = TreeCache([900], 2, 1, d, 16, dtype, new=[tokens], seed=d, max_pages=4096 if split else None)
    assert cut(c) == (split or (dtype, d, tokens) == ("fp32", 128, 4))  # (whose tiles are large)
    growing(c, 900, d)
    Q, O, lse = run_tree(c, Q=(c.normal(tokens, 2, d).abs() * 0.5 + 0.5).to(DTYPES[dtype]))
    check_grown(O, lse, *c.want_tree(Q), dtype, d)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [[1, 3, 2, 0, 5], [1, 40, 64, 0, 31]])
@pytest.mark.parametrize("split", [False, True])
def test_large_logits(dtype, d, kind, new, split):
    c = TreeCache([1, 300, 64, 0, 31], 4, 2, d, 16, dtype, new=new, seed=d, max_pages=4096 if split else None)
    assert cut(c) == split
    fill(c, kind)
    Q, O, lse = run_tree(c, Q=queries(c, c.T))
    check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_keys_at_minus_infinity_have_no_weight(dtype, d):
    # one sequence has nothing else: as if it saw nothing
    c = TreeCache([90, 33], 4, 2, d, 16, dtype, new=[40, 20], seed=4)
    c.K_cache[int(c.table[0, 0, 1]), :, 3, 0] = float("-inf")
    for i in c.table[1, 0][:3]:
        c.K_cache[int(i), :, :, 0] = float("-inf")
    Q = c.normal(c.T, 4, d)
    Q[..., 0] = Q[..., 0].abs() + 0.01
    Q, O, lse = run_tree(c, Q=Q)
    wO, wl = c.want_tree(Q)
    wO[40:], wl[40:] = 0.0, float("-inf")
    assert torch.equal(O[40:].double().cpu(), wO[40:]) and torch.equal(lse[40:].double().cpu(), wl[40:])
    check(O[:40], lse[:40], wO[:40], wl[:40], dtype)
