"""Sequences that go on by many pages at once: which entries of a long row are fresh, and that it takes no longer for rows being long."""
import numpy as np
import pytest
import torch

from paper_2512_13368_amd import binding as B
from test_gpu_fork import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,width,grow", [(3, 200, 1500), (70, 150, 900), (5, 2100, 16700)])
@pytest.mark.parametrize("seed", range(3))
def test_fresh_pages_among_pages_that_are_kept(S, width, grow, seed):
    # tables full of pages behind short lengths: some held once, which stay, some by others too, which are replaced, some none
    rng = np.random.default_rng(seed)
    n_pages = 2 * S * width + 100
    order = [int(x) for x in rng.permutation(n_pages)]
    refs, table = [0] * n_pages, []
    for _ in range(S):
        row = []
        kind = rng.choice(["all", "none", "mixed", "blocks"])
        for i in range(width):
            p = order.pop()
            there = {"all": True, "none": False, "mixed": rng.random() < 0.5, "blocks": (i // 70) % 2 == 0}[str(kind)]
            row.append(p if there else int(rng.choice([-1, n_pages])))
            if there:
                refs[p] = int(rng.choice([1, 1, 2]))
        table.append(row)
    lens = [int(x) for x in rng.integers(0, 8 * width, S)]
    lens[0] = 5
    run(table, lens, refs, list(range(S)), 8, grow)
    run(table, lens, refs, [int(x) for x in rng.integers(0, S, S + 2)], 8, grow)


def test_requests_of_several_sweeps():
    # one row that asks for more pages than a sweep looks at, between pages that are held
    width, n_pages = 20000, 60000
    table = [[int(i) if i % 3 == 0 else -1 for i in range(width)]]
    refs = [0] * n_pages
    for p in table[0]:
        if p >= 0:
            refs[p] = 1
    run(table, [9], refs, [0], 8, 8 * width)


def test_long_rows_take_no_longer():
    """As many pages, in 64 rows and in 8: a request that looked for its entry from the row's first on would take several times as long."""
    def least(S, width):
        p = B.PagedParams(S=S, T=1, H=1, G=1, d=8, page=8, n_pages=2 * S * width, max_pages=width)
        i32 = dict(dtype=torch.int32, device="cuda")
        table, n, refs = torch.full((S, width), -1, **i32), torch.zeros(S, **i32), torch.zeros(p.n_pages, **i32)
        parent = torch.arange(S, **i32)
        print(f"fork {p}", flush=True)
        out = B.kv_fork(p, parent, table, n, refs, grow=8 * width)
        ws = torch.empty(B.fork_workspace_bytes(p, S), dtype=torch.uint8, device="cuda")
        times = []
        for _ in range(20):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            B.kv_fork(p, parent, table, n, refs, grow=8 * width, new_table=out[0], new_len=out[1], new_refs=out[2], copies=out[3], missing=out[4], ws=ws)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        assert torch.equal(out[0].flatten(), torch.arange(S * width, **i32)) and int(out[4]) == 0
        print(f"{min(times):.3f} ms", flush=True)
        return min(times)

    assert least(8, 8192) < 2 * least(64, 1024)
