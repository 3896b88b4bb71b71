"""Beam search's selection where a row's largest logit is far from 0: such a row's sum is that of differences, and what is ruled out, or lies
behind the row's end, has no part in it."""
import numpy as np
import pytest
import torch

from paper_2512_13368_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def want_best(logits, score, K):
    """(parent, token, score, bound on the score's error) by the definition in 64 bits, of differences to a row's largest logit."""
    b_, w_ = score.shape
    x = logits.double().numpy().reshape(b_, w_, -1)
    out = np.full((b_, K), -1), np.full((b_, K), -1), np.full((b_, K), -np.inf), np.zeros((b_, K))
    for b in range(b_):
        rows = []
        for w in range(w_):
            c = float(score[b, w])
            r = np.where(np.isnan(x[b, w]), -np.inf, x[b, w])
            m = r.max()
            if not np.isfinite(m):
                continue
            with np.errstate(under="ignore"):
                to = c + ((r - m) - np.log(np.exp(r - m).sum()))
            # rounded once to 32 bits; exponentials to 1.1e-12, of which a sum and its log keep no more; three operations in 64 bits
            bound = np.abs(to) * 2.0**-24 + 4e-12 + (abs(c) + np.abs(r - m)) * 2.0**-51
            rows.append((to, r, np.arange(r.size), np.full(r.size, w), bound))
        to, r, v, w, bound = (np.concatenate(c) for c in zip(*rows))
        ok = to > -np.inf
        to, r, v, w, bound = to[ok], r[ok], v[ok], w[ok], bound[ok]
        at = np.lexsort((v, -r, w, -to))[:K]
        n = len(at)
        out[0][b, :n], out[1][b, :n], out[2][b, :n], out[3][b, :n] = b * w_ + w[at], v[at], to[at], bound[at]
    return out


def run(logits, score, K):
    b, w, v = logits.shape
    p = B.BeamParams(B=b, W=w, K=K, V=v, dtype=B.F32 if logits.dtype == torch.float32 else B.BF16)
    print(f"beam {p}", flush=True)
    got = [x.cpu().numpy() for x in B.beam_select(p, logits.view(b * w, v).cuda(), score.cuda())]
    want = want_best(logits, score, K)
    assert np.array_equal(got[0], want[0]), "parents"
    assert np.array_equal(got[1], want[1]), "items"
    fine = np.isfinite(want[2])
    assert np.array_equal(got[2][~fine], want[2][~fine].astype(np.float32))
    assert (np.abs(got[2][fine].astype(np.float64) - want[2][fine]) <= want[3][fine]).all(), "scores"


def rows_about(top, v, dtype, seed):
    """Four rows of v logits: one at `top` and nothing else; all at `top`; some a unit or more below it among ordinary and ruled out ones;
    ordinary ones of a few items, all others at `top` below 0."""
    g = torch.Generator().manual_seed(seed)
    top = torch.tensor(top).to(DT[dtype]).float()
    x = torch.full((4, v), float("-inf"))
    x[0, v // 3] = top
    x[1] = top
    x[2] = torch.randn(v, generator=g)
    x[2, ::5] = top * (1.0 - 2.0**-6 * torch.randint(0, 3, (len(range(0, v, 5)),), generator=g))
    x[2, 1::7] = float("nan")
    x[2, 3::7] = float("-inf")
    x[3] = -top.abs()
    x[3, v // 4:v // 4 + 5] = torch.randn(5, generator=g)
    return x.to(DT[dtype])


TOPS = [5e3, 1e9, 3e9, 1e10, 1e11, 1e15, 1e30, 3.3e38]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("top", TOPS + [-x for x in TOPS])
@pytest.mark.parametrize("v", [37, 1501, 3000, 50021])
def test_rows_far_from_zero(dtype, top, v):
    logits = torch.stack([rows_about(top, v, dtype, v + i) for i in range(2)])
    score = -torch.rand(2, 4, generator=torch.Generator().manual_seed(v)) * 8
    run(logits, score, 6)
    run(logits, score, 33)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("top", [3e9, -1e10, 1e15])
def test_long_runs_far_from_zero(dtype, top):
    # rows that are long for a workgroup, some of whose pieces lie near 0
    logits = torch.stack([torch.cat([rows_about(top, 150001, dtype, i), rows_about(top, 150001, dtype, i + 9)]) for i in range(3)])
    logits[:, 5, 20000:60000] = torch.randn(40000, generator=torch.Generator().manual_seed(1)).to(DT[dtype])
    run(logits, -torch.rand(3, 8, generator=torch.Generator().manual_seed(2)) * 8, 16)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("v", [300, 20000])
def test_beams_far_from_zero_are_told_apart(dtype, v):
    # the same differences at other places: what a beam has come to decides, to the last bit of 32
    g = torch.Generator().manual_seed(v)
    few = torch.randint(0, 2, (v,), generator=g).float() * 2.0**33
    logits = torch.stack([few - 2.0**40, few + 2.0**39, few, few - 2.0**39])[None].to(DT[dtype])
    assert torch.equal(logits[0, 0].float() + 2.0**40, few)
    score = torch.tensor([[-3.0, -3.0 + 2.0**-22, -3.0 + 2.0**-21, -3.0 - 2.0**-22]])
    run(logits, score, 40)
