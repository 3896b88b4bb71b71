"""Beam search's selection against its definition in 64 bits: items and beams are whole numbers, and equal."""
import numpy as np
import pytest
import torch

from paper_2512_13368_amd import binding as B
from tree_util import want_beam

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def run(logits, score, K, ended=None, eos=-1, dev=None):
    """logits [B, W, V] and score [B, W] on the CPU; dev: the rows on the GPU, where they are not simply those."""
    b, w, v = logits.shape
    dtype = B.F32 if logits.dtype == torch.float32 else B.BF16
    p = B.BeamParams(B=b, W=w, K=K, V=v, dtype=dtype, eos=eos)
    print(f"beam {p}", flush=True)
    guard = [torch.full((b * K + 8,), x, dtype=t, device="cuda") for x, t in ((77, torch.int32), (77, torch.int32), (77.0, torch.float32), (True, torch.bool))]
    out = [g[:-8].view(b, K) for g in guard]
    rows = logits.view(b * w, v).cuda() if dev is None else dev
    B.beam_select(p, rows, score.cuda(), ended=None if ended is None else ended.cuda(), parent=out[0], token=out[1], out_score=out[2], out_ended=out[3])
    torch.cuda.synchronize()
    assert all((g[-8:] == x).all() for g, x in zip(guard, (77, 77, 77.0, True))), "something behind an output was written"
    want = want_beam(logits, score, K, ended, eos)
    got = [x.cpu().numpy() for x in out]
    assert np.array_equal(got[0], want[0]), "parents"
    assert np.array_equal(got[1], want[1]), "items"
    assert np.array_equal(got[3], want[3]), "ends"
    fine = np.isfinite(want[2])
    assert np.array_equal(got[2][~fine], want[2][~fine].astype(np.float32))
    # rounded once from 64 bits: half a unit of fp32
    assert (np.abs(got[2][fine] - want[2][fine]) <= np.abs(want[2][fine]) * 2.0 ** -24 + 1e-30).all()
    return out


def inputs(b, w, v, dtype, seed, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(b, w, v, generator=g) * scale).to(DT[dtype]), -torch.rand(b, w, generator=g) * 10


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("b,w,k,v", [(1, 1, 1, 1), (1, 1, 5, 3), (3, 4, 4, 7), (2, 3, 64, 50), (5, 8, 8, 1000), (2, 64, 64, 333), (2, 5, 9, 2047), (2, 5, 9, 2049),
                                     (1, 4, 16, 40001), (3, 2, 7, 16384), (1, 33, 40, 8193), (70, 4, 8, 5001), (1, 1, 32, 300001)])
def test_best_continuations(dtype, b, w, k, v):
    run(*inputs(b, w, v, dtype, v + w), k)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("v,pad,at", [(1001, 1, 0), (1001, 1, 1), (999, 1003, 3), (4099, 4160, 5), (16385, 16387, 1)])
def test_rows_may_begin_at_any_element(dtype, v, pad, at):
    logits, score = inputs(3, 4, v, dtype, v)
    pad = max(pad, v)
    wide = torch.full((12 * pad + at + 8,), float("inf"), dtype=DT[dtype])  # what lies between rows is not read into anything
    rows = wide[at:at + 12 * pad].view(12, pad)
    rows[:, :v] = logits.view(12, v)
    dev = wide.cuda()[at:at + 12 * pad].view(12, pad)[:, :v]
    run(logits, score, 6, dev=dev)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("v", [40, 3000, 40000])
def test_equal_logits_go_by_item_and_equal_beams_by_beam(dtype, v):
    run(torch.zeros(2, 3, v, dtype=DT[dtype]), torch.zeros(2, 3), 64)
    same = inputs(2, 1, v, dtype, v)[0].expand(2, 5, v).contiguous()
    run(same, torch.full((2, 5), -1.5), 17)
    few = (torch.randint(0, 3, (2, 4, v), generator=torch.Generator().manual_seed(1)) - 1).to(DT[dtype])  # many of each value, 0 and -0 too
    few[:, :, ::2] = few[:, :, ::2] * -1.0
    run(few, inputs(2, 4, v, dtype, 1)[1], 30)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_large_logits_in_the_same_places(dtype):
    # many large logits where one thread's loads lie, in order and in reverse
    v = 40000
    logits, score = inputs(2, 2, v, dtype, 7, scale=0.1)
    logits[0, 0, ::256 * 8] += 20.0
    logits[1, 1, :8] += 30.0
    logits[0, 1] = torch.arange(v).to(DT[dtype]) / 1000
    logits[1, 0] = -torch.arange(v).to(DT[dtype]) / 1000
    run(logits, score, 64)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("v", [30, 5000, 50000])
def test_items_and_beams_that_are_ruled_out(dtype, v):
    logits, score = inputs(6, 4, v, dtype, v)
    inf, nan = float("inf"), float("nan")
    logits[0, 0] = -inf                       # a row of nothing
    logits[0, 1, 3:] = -inf                   # three items left
    logits[1] = -inf                          # a history without a candidate
    logits[2, 0, 5] = nan                     # counts as ruled out
    logits[2, 1] = nan
    logits[2, 2, 7] = inf                     # such a row has no candidate
    score[3] = torch.tensor([-inf, 0.0, nan, -inf])  # as at a search's first step: one beam that counts
    score[4, 1] = inf
    logits[5, :, 2:] = -inf
    run(logits, score, 8)
    run(logits, score, 64)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("flag", [torch.bool, torch.uint8])
def test_beams_at_their_end_go_on_in_one_way(dtype, flag):
    for v, eos in ((20, 0), (3000, 2999), (20000, 123)):
        logits, score = inputs(5, 6, v, dtype, v)
        ended = torch.rand(5, 6, generator=torch.Generator().manual_seed(v)) < 0.5
        ended[0], ended[1] = True, False
        score[2, 0], ended[2, 0] = float("-inf"), True
        score[3], ended[3, :2] = -2.5, True  # two ends of the same score
        logits[:, 1, eos] += 9.0
        run(logits, score, 6, ended=ended.to(flag), eos=eos)
        run(logits, score, 40, ended=ended.to(flag), eos=eos)


def test_logits_and_scores_of_any_size():
    for scale in (1e-30, 1e-3, 100.0, 1e4, 1e30):
        logits, score = inputs(3, 3, 3000, "fp32", 5, scale=scale)
        run(logits, score, 12)
    logits, score = inputs(3, 3, 3000, "fp32", 6)
    run(logits, score * 1e-6 - 50.0, 12)
    run(logits, torch.tensor([[1e30, 1e30, -1e30]] * 3), 12)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_two_calls_give_the_same_bits(dtype):
    logits, score = inputs(16, 8, 50021, dtype, 3)
    first = [x.clone() for x in run(logits, score, 16)]
    for a, b in zip(first, run(logits, score, 16)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("b,w,k,v", [(300, 2, 3, 700), (300, 1, 4, 5000), (300, 6, 4, 1000), (520, 3, 8, 2731), (513, 1, 2, 3)])
def test_many_histories(dtype, b, w, k, v):
    run(*inputs(b, w, v, dtype, b + v), k)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("v", [600, 9000, 100003])
def test_logits_below_zero(dtype, v):
    # as log-probabilities are; then with a few NaN of either sign and +-0 among them
    g = torch.Generator().manual_seed(v)
    logits = (-torch.rand(2, 3, v, generator=g) * 18 - 0.125).to(DT[dtype])
    score = -torch.rand(2, 3, generator=g)
    run(logits, score, 20)
    logits[0, 0, 5::97], logits[0, 1, 3::89], logits[1, 2, 7::101] = float("nan"), -float("nan"), -0.0
    logits[1, 0, v // 2] = 0.0
    run(logits, score, 20)
    run(logits * 6.0, score, 20)
