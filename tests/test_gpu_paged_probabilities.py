"""What rounding costs where the cache's bf16 values are multiplied by probabilities.  Queries and keys are multiples of 1/4 up to 2, so
that logits are exact in fp32 and all that is left is the probabilities' way to the values."""
import numpy as np
import pytest
import torch

from paged_util import DTYPES, Cache
from paper_2512_13368_amd import binding as B
from test_gpu_paged import run_decode, run_prompt

pytestmark = pytest.mark.gpu


def coarse(c, *shape):
    return torch.from_numpy(c.rng.integers(-8, 9, shape) / 4.0).to(DTYPES[c.dtype])


def coarse_keys(c):
    held = ~torch.isnan(c.K_cache)
    c.K_cache[held] = coarse(c, int(held.sum()))


def check_fine(c, O, Q, rows):
    """|O - ref| <= 2^-8 |ref| + A (2^-17 + (n + 16) 2^-24): half a unit of bf16 for the result, and, of A = sum p |V| over n keys, two bf16
    terms a probability, a rounding in 32 bits for each key that is added, for logits of up to 16 in units of the exponent."""
    worst, V = -1.0, c.V_cache
    for row, s, pos in rows:
        for h in range(c.H):
            c.V_cache = V
            want, _ = c.attend(Q[row, h], s, h, pos)
            c.V_cache = V.abs()
            size, _ = c.attend(Q[row, h], s, h, pos)
            off = (O[row, h].double().cpu() - want).abs() - 2.0**-8 * want.abs() - size * (2.0**-17 + (pos + 17) * 2.0**-24)
            worst = max(worst, float(off.max()))
    c.V_cache = V
    assert worst <= 0, f"off by {worst:.3g} beyond the bound"


@pytest.mark.parametrize("d,page", [(8, 8), (16, 16), (32, 32), (64, 16), (128, 64)])
@pytest.mark.parametrize("split", [False, True])
def test_decode_keeps_its_probabilities(d, page, split):
    c = Cache([1, 2, 5, 33, 300], 4, 2, d, page, "bf16", seed=d, max_pages=8192 if split else None, scale=0.5 * d**-0.5)
    assert (B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0) == split
    coarse_keys(c)
    Q, O, _ = run_decode(c, Q=coarse(c, 5, 4, d))
    check_fine(c, O, Q, [(s, s, n - 1) for s, n in enumerate(c.kv_len)])


@pytest.mark.parametrize("d,page", [(8, 8), (16, 16), (32, 32), (64, 16), (128, 64)])
@pytest.mark.parametrize("long", [False, True])
def test_few_new_tokens_keep_their_probabilities(d, page, long):
    kv = [3, 40, 2100] if long else [3, 40, 210]
    c = Cache(kv, 4, 2, d, page, "bf16", new=[3, 2, 7], seed=d, scale=0.5 * d**-0.5)
    assert (B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0) == long
    coarse_keys(c)
    Q, O, _ = run_prompt(c, Q=coarse(c, c.T, 4, d))
    check_fine(c, O, Q, [(int(c.cu[s]) + i, s, n - c.new[s] + i) for s, n in enumerate(kv) for i in range(c.new[s])])
