"""Forked sequences and copied pages against their definition on whole numbers."""
import numpy as np
import pytest
import torch

from paper_2512_13368_amd import binding as B
from tree_util import want_fork

pytestmark = pytest.mark.gpu


def state(S, page, width, n_pages, seed, shared=True, junk=False):
    """Page tables of S sequences with refs that count them, some whole pages shared."""
    rng = np.random.default_rng(seed)
    lens = [int(x) for x in rng.integers(0, width * page + 1, S)]
    order = list(rng.permutation(n_pages))
    table, refs = [], [0] * n_pages
    for s in range(S):
        held = min(width, -(-lens[s] // page) + int(rng.integers(0, 2)))  # at times a page more than it needs
        row = []
        for i in range(held):
            other = int(rng.integers(0, max(s, 1)))
            if shared and s and rng.random() < 0.5 and i < lens[s] // page and i < lens[other] // page and table[other][i] >= 0:
                row.append(table[other][i])
            else:
                row.append(int(order.pop()) if order else -1)
        table.append(row + [-1] * (width - held))
    if junk:
        for s in range(S):
            table[s][int(rng.integers(0, width))] = int(rng.choice([-1, n_pages, 2**31 - 1, -2**31]))
    for row in table:
        for p in row:
            if 0 <= p < n_pages:
                refs[p] += 1
    return table, lens, refs, rng


def run(table, lens, refs, parent, page, grow, max_len=0, ws=None):
    S, width, n_pages, N = len(table), len(table[0]), len(refs), len(parent)
    p = B.PagedParams(S=S, T=1, H=1, G=1, d=8, page=page, n_pages=n_pages, max_pages=width, max_len=max_len)

    def dev(x):
        return torch.tensor(x, dtype=torch.int32).cuda()

    print(f"fork {p} N={N} grow={grow}", flush=True)
    guard = [torch.full((n + 8,), 77, dtype=torch.int32, device="cuda") for n in (N * width, N, n_pages, N * 3, 1)]
    shapes = [(N, width), (N,), (n_pages,), (N, 3), (1,)]
    out = [g[:-8].view(s) for g, s in zip(guard, shapes)]
    given = [dev(x) for x in (parent, table, lens, refs)]
    B.kv_fork(p, *given, grow=grow, new_table=out[0], new_len=out[1], new_refs=out[2], copies=out[3], missing=out[4], ws=ws)
    torch.cuda.synchronize()
    assert all((g[-8:] == 77).all() for g in guard), "something behind an output was written"
    for g, x in zip(given, (parent, table, lens, refs)):
        assert g.cpu().tolist() == x, "an input changed"
    want = want_fork(table, lens, refs, parent, page, p.capacity, grow)
    for name, g, w in zip(("table", "len", "refs", "copies", "missing"), out, want):
        assert g.cpu().tolist() == w, name
    return out


@pytest.mark.parametrize("S,N,page,width", [(1, 1, 8, 1), (1, 4, 8, 7), (4, 4, 16, 9), (7, 33, 32, 70), (64, 64, 16, 300), (300, 515, 8, 40), (5, 1, 256, 3)])
@pytest.mark.parametrize("grow", [0, 1, 40])
def test_forked_tables(S, N, page, width, grow):
    table, lens, refs, rng = state(S, page, width, 2 * (S + N) * width, S + N + grow)
    parent = [int(x) for x in rng.integers(0, S, N)]
    run(table, lens, refs, parent, page, grow)


@pytest.mark.parametrize("S,N", [(6, 6), (40, 90)])
def test_dropped_sequences_and_parents_that_are_none(S, N):
    table, lens, refs, rng = state(S, 8, 20, 2 * (S + N) * 20, 3)
    parent = [int(x) for x in rng.choice([-1, 0, 1, S, S - 1, -2**31, 2**31 - 1], N)]
    run(table, lens, refs, parent, 8, 1)
    run(table, lens, refs, [-1] * N, 8, 5)


def test_the_same_sequences_go_on_and_make_room():
    # parents in place: nothing is copied, pages behind the lengths go back, pages for 20 more positions come
    table, lens, refs, _ = state(9, 8, 12, 500, 4, shared=False)
    lens = [max(0, n - 9) for n in lens]
    out = run(table, lens, refs, list(range(9)), 8, 20)
    assert (out[3][:, 0] == -1).all() and int(out[4]) == 0


@pytest.mark.parametrize("spare", [0, 1, 5, 20])
def test_too_few_free_pages(spare):
    table, lens, refs, rng = state(8, 8, 10, 300, 5)
    held = 0
    for p in range(300):  # somebody else holds all others but a few
        if refs[p] == 0:
            held += 1
            refs[p] = 1 if held > spare else 0
    parent = [0, 0, 0, 1, 1, 5, 5, 5, 5, 2, 3]
    run(table, lens, refs, parent, 8, 12)


def test_partly_filled_pages_that_several_hold_are_copied_for_all():
    # four sequences with one table, made by hand: the page that all hold partly filled stays nobody's and is not given out
    table = [[3, 5, 1, -1]] * 4
    refs = [0] * 6
    for p in (3, 5, 1):
        refs[p] = 4
    out = run([list(r) for r in table], [20] * 4, refs, [0, 1, 2, 3], 8, 1)
    # (three pages are free: the fourth goes without a copy)
    assert out[3][:, 0].tolist() == [1, 1, 1, -1] and int(out[4]) == 1
    # two share one that only one goes on from
    run([[0, 1], [0, 1]], [12, 12], [2, 2, 0, 0, 0, 0], [1], 8, 1)


def test_entries_that_are_no_pages_and_capacity():
    for seed in range(4):
        table, lens, refs, rng = state(12, 8, 15, 900, seed, junk=True)
        lens[0], lens[1] = -5, 10**9
        parent = [int(x) for x in rng.integers(-1, 13, 30)]
        run(table, lens, refs, parent, 8, 9)
        run(table, lens, refs, parent, 8, 9, max_len=61)
        run(table, lens, refs, parent, 8, 2**31 - 1)


def test_fork_of_many_pages():
    # more pages than one sweep of the search for free ones takes, all free ones at the end
    table, lens, refs, rng = state(20, 8, 30, 5000, 8)
    n = 70001
    refs = refs + [1] * (n - 5000 - 50) + [0] * 50
    run(table, lens, [max(r, 1) if i < 5000 else r for i, r in enumerate(refs)], [int(x) for x in rng.integers(0, 20, 60)], 8, 1)


@pytest.mark.parametrize("dtype,G,d,page", [(torch.float32, 1, 8, 8), (torch.float32, 3, 128, 16), (torch.bfloat16, 2, 64, 32),
                                            (torch.bfloat16, 8, 128, 256), (torch.bfloat16, 4, 16, 64)])
def test_copied_pages(dtype, G, d, page):
    rng = np.random.default_rng(d)
    n_pages, n = 40, 15
    ids = rng.permutation(n_pages)
    copies = [[int(ids[i]), int(ids[20 + i]), int(rng.integers(0, page + 1))] for i in range(n)]
    copies += [[-1, 3, 5], [int(ids[0]), n_pages, 4], [int(ids[1]), int(ids[1]), 8], [int(ids[2]), int(ids[38]), 2**31 - 1], [int(ids[3]), int(ids[39]), -2]]
    p = B.PagedParams(S=1, T=1, H=G, G=G, d=d, page=page, n_pages=n_pages, max_pages=1, dtype=B.F32 if dtype == torch.float32 else B.BF16)
    K, V = (torch.randn(n_pages, G, page, d).to(dtype) for _ in range(2))
    Kc, Vc = K.cuda(), V.cuda()
    print(f"copy {p}", flush=True)
    B.kv_copy_pages(p, torch.tensor(copies, dtype=torch.int32).cuda(), Kc, Vc)
    torch.cuda.synchronize()
    for was, got in ((K, Kc), (V, Vc)):
        want = was.clone()
        for a, b, rows in copies:
            if 0 <= a < n_pages and 0 <= b < n_pages and a != b:
                rows = max(0, min(rows, page))
                want[b, :, :rows] = was[a, :, :rows]
        assert torch.equal(got.cpu(), want)
