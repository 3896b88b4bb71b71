"""What rounding costs drafted trees of bf16: an output is off by its own rounding, however many rows a tree has.  Queries and keys are
multiples of 1/4 up to 2, so that logits are exact in fp32 and all that is left is the probabilities' way to the values."""
import pytest

from paper_2512_13368_amd import binding as B
from test_gpu_paged_probabilities import coarse, coarse_keys
from test_gpu_tree import run_tree
from tree_util import TreeCache

pytestmark = pytest.mark.gpu

DIMS = [8, 16, 32, 64, 128]


def check_fine(c, O, Q):
    """|O - ref| <= 2^-8 |ref| + A (2^-17 + (n + 48) 2^-24): half a unit of bf16 for the result, and, of A = sum p |V| over n keys, two bf16
    terms a probability, a rounding in 32 bits for each key that is added, 32 for an exponent's argument of up to 32, and 16 for the four
    factors that a sum meets (a reference moved, wavefronts joined, parts joined, the division), each an exponential of a unit and products."""
    worst, V = -1.0, c.V_cache
    for s, new in enumerate(c.new):
        for i in range(new):
            row = int(c.cu[s]) + i
            for h in range(c.H):
                c.V_cache = V
                want, _ = c.attend_tree(Q[row, h], s, i, h)
                c.V_cache = V.abs()
                size, _ = c.attend_tree(Q[row, h], s, i, h)
                off = (O[row, h].double().cpu() - want).abs() - 2.0**-8 * want.abs() - size * (2.0**-17 + (c.kv_len[s] + 48) * 2.0**-24)
                worst = max(worst, float(off.max()))
    c.V_cache = V
    assert worst <= 0, f"off by {worst:.3g} beyond the bound"


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("H,new,kv", [(2, [3, 5, 1], [300, 90, 200]), (2, [40, 3, 64], [300, 150, 260]), (6, [64, 50, 64], [300, 70, 200])])
@pytest.mark.parametrize("window", [0, 150])
def test_trees_keep_their_probabilities(d, H, new, kv, window):
    c = TreeCache(kv, H, 1, d, 16, "bf16", new=new, seed=d, window=window, scale=0.5 * d**-0.5)
    assert B.paged_workspace_bytes(c.p, B.WS_TREE) == 0
    coarse_keys(c)
    Q, O, _ = run_tree(c, Q=coarse(c, c.T, H, d))
    check_fine(c, O, Q)


@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("H,new", [(2, [3, 7]), (2, [40, 20]), (6, [64, 50])])
def test_so_do_walks_that_are_split(d, H, new):
    # logits that leave few keys with weight
    c = TreeCache([1300, 700], H, 1, d, 16, "bf16", new=new, seed=d, max_pages=1024, scale=d**-0.5)
    assert B.paged_workspace_bytes(c.p, B.WS_TREE) > 0
    coarse_keys(c)
    Q, O, _ = run_tree(c, Q=coarse(c, c.T, H, d))
    check_fine(c, O, Q)
