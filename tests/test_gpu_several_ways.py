"""Drafted trees, forked pages and beams together, as a server uses them; long and wide calls; streams, graphs and offsets beyond 32 bits."""
import numpy as np
import pytest
import torch

from paged_util import DTYPES, TOL, Cache, check
from paper_2512_13368_amd import binding as B
from test_gpu_beam import inputs, run as run_beam
from test_gpu_fork import run as run_fork, state
from test_gpu_paged import rope, rotated
from test_gpu_tree import run_tree
from tree_util import TreeCache, signed, tree_masks, want_beam

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# ---- a beam search ----


class Model:
    """One attention layer and its logits: what a sequence's last item attends to is a function of its items alone."""

    def __init__(self, H, G, d, items, cap, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        self.H, self.G, self.d, self.dt = H, G, d, DTYPES[dtype]
        self.q, self.k, self.v = (torch.randn(items, n, d, generator=g).to(self.dt) for n in (H, G, G))
        self.out = torch.randn(H * d, items, generator=g)
        self.cos, self.sin = rope(cap, d)
        self.rope = self.cos.cuda(), self.sin.cuda()
        self.dev = [x.cuda() for x in (self.q, self.k, self.v, self.out)]

    def rows(self, tokens):
        return [x[tokens.long()] for x in self.dev[:3]]

    def attend(self, tokens):
        """The last item's attention in 64 bits; keys and queries rounded as the cache holds them."""
        t = torch.tensor(tokens)
        n = len(tokens)
        k = torch.stack([rotated(self.k[t[i]], self.cos[i], self.sin[i]) for i in range(n)]).to(self.dt).double()
        q = rotated(self.q[t[-1]], self.cos[n - 1], self.sin[n - 1]).to(self.dt).double()
        v, share, out = self.v[t].double(), self.H // self.G, []
        for h in range(self.H):
            x = (k[:, h // share] @ q[h]) * self.d ** -0.5
            out.append(torch.softmax(x, 0) @ v[:, h // share])
        return torch.stack(out)


@pytest.mark.parametrize("dtype,d,W,page", [("fp32", 32, 3, 8), ("bf16", 64, 8, 16), ("bf16", 128, 1, 8)])
def test_a_beam_search_over_one_cache(dtype, d, W, page):
    H, G, items, lengths, steps, width = 4, 2, 700, [1, 37, 16, 90], 12, 15
    S = len(lengths)
    model = Model(H, G, d, items, width * page, dtype, W)
    n_pages = S * (W + 12) + 40 + S * W * 4
    p = B.PagedParams(S=S, T=sum(lengths), H=H, G=G, d=d, page=page, n_pages=n_pages, max_pages=width, dtype=B.F32 if dtype == "fp32" else B.BF16)
    caches = [torch.full((n_pages, G, page, d), float("nan"), dtype=model.dt, device="cuda") for _ in range(2)]
    rng = np.random.default_rng(W)
    held = [[int(x) for x in rng.integers(0, items, n)] for n in lengths]
    refs = i32([0] * n_pages)
    # pages for the prompts from a fork of sequences that hold nothing yet
    table, _, refs, _, missing = B.kv_fork(p, i32(list(range(S))), i32([[-1] * width] * S), i32([0] * S), refs, grow=max(lengths))
    assert int(missing) == 0
    cu = i32(np.concatenate([[0], np.cumsum(lengths)]).tolist())
    kv_len = i32(lengths)
    q, k, v = model.rows(torch.tensor(sum(held, [])).cuda())
    q = B.kv_append(p, k, v, *caches, table, cu, kv_len, Q=q, rope=model.rope)
    O, _ = B.attn_prompt(p, q, *caches, table, cu, kv_len)
    last = O[(cu[1:] - 1).long()]
    score, ended = torch.zeros(S, 1), torch.zeros(S, 1, dtype=torch.bool)
    for step in range(steps):
        now = score.shape[1]  # the first step goes from a beam each to W
        logits = last.float().flatten(1) @ model.dev[3]
        bp = B.BeamParams(B=S, W=now, K=W, V=items, dtype=B.F32, eos=5)
        parent, token, new_score, new_ended = B.beam_select(bp, logits, score.cuda(), ended=ended.cuda())
        want = want_beam(logits.cpu().view(S, now, -1), score, W, ended, 5)
        for got, w in zip((parent, token, new_ended), (want[0], want[1], want[3])):
            assert np.array_equal(got.cpu().numpy(), w), f"step {step}"
        held = [held[a] + [b] for a, b in zip(parent.flatten().tolist(), token.flatten().tolist())]
        score, ended = new_score.cpu(), new_ended.cpu()
        here = B.PagedParams(**{**p.__dict__, "S": S * now, "T": S * now})
        table, kv_len, refs, copies, missing = B.kv_fork(here, parent.view(-1), table, kv_len, refs, grow=1)
        assert int(missing) == 0
        B.kv_copy_pages(here, copies, *caches)
        N = S * W
        there = B.PagedParams(**{**p.__dict__, "S": N, "T": N})
        kv_len = kv_len + 1
        q, k, v = model.rows(token.view(-1))
        one = torch.arange(N + 1, dtype=torch.int32, device="cuda")
        q = B.kv_append(there, k, v, *caches, table, one, kv_len, Q=q, rope=model.rope)
        last, _ = B.attn_decode(there, q, *caches, table, kv_len)
        ref = torch.stack([model.attend(h) for h in held])
        off = (last.double().cpu() - ref).abs() - TOL[dtype] * (ref.abs() + ref.pow(2).mean().sqrt())
        assert float(off.max()) <= 0, f"step {step}: off by {float(off.max()):.3g} beyond the bound"
        # every entry is counted, and no page that is written next has two holders
        count = torch.bincount(table[table >= 0].long(), minlength=n_pages)
        assert torch.equal(count, refs.long())
        tails = [int(table[n, int(kv_len[n]) // page]) for n in range(N) if int(kv_len[n]) % page]
        assert len(set(tails)) == len(tails)


# ---- drafts, checked and taken over ----


@pytest.mark.parametrize("dtype,H,G,d", [("fp32", 4, 2, 32), ("bf16", 8, 2, 64), ("bf16", 8, 8, 128)])
def test_drafts_that_are_accepted_are_as_if_appended(dtype, H, G, d):
    rng = np.random.default_rng(d)
    new, past = [1, 12, 40, 64, 5], [30, 100, 0, 333, 17]
    parents = [[int(rng.integers(-1, i)) if i else -1 for i in range(n)] for n in new]
    c = TreeCache([a + b for a, b in zip(new, past)], H, G, d, 16, dtype, new=new, masks=[tree_masks(u) for u in parents], seed=d)
    paths = []
    for s, n in enumerate(new):  # the way down to the last token
        path, at = [], n - 1
        while at >= 0:
            path.append(at)
            at = parents[s][at]
        paths.append(path[::-1])
    Kc, Vc, table, cu, kv_len = c.dev()
    plain = [Kc.clone(), Vc.clone()]
    q, k, v = (c.normal(c.T, n, d).cuda() for n in (H, G, G))
    turn = [x.cuda() for x in rope(c.cap, d)]
    q_rot = B.kv_append_tree(c.p, k, v, Kc, Vc, table, cu, kv_len, c.mask(), Q=q, rope=turn)
    lse = torch.empty(c.T, H, device="cuda")
    O, _ = B.attn_tree(c.p, q_rot, Kc, Vc, table, cu, kv_len, c.mask(), lse=lse)
    width = max(len(x) for x in paths)
    new_len = B.kv_accept(c.p, i32([x + [-1] * (width - len(x)) for x in paths]), Kc, Vc, table, cu, kv_len)
    assert new_len.tolist() == [a + len(x) for a, x in zip(past, paths)]
    # the same tokens as a prompt
    rows = torch.tensor([int(c.cu[s]) + i for s, x in enumerate(paths) for i in x]).cuda()
    p = B.PagedParams(**{**c.p.__dict__, "T": len(rows)})
    at = i32(np.concatenate([[0], np.cumsum([len(x) for x in paths])]).tolist())
    q_plain = B.kv_append(p, k[rows], v[rows], *plain, table, at, new_len, Q=q[rows], rope=turn)
    assert torch.equal(q_plain, q_rot[rows])
    bits = torch.int32 if dtype == "fp32" else torch.int16
    for s, n in enumerate(new_len.tolist()):
        j = torch.arange(n, device="cuda")
        ids = table[s].long()[j // 16]
        for got, want in zip((Kc, Vc), plain):
            assert torch.equal(got[ids, :, j % 16].view(bits), want[ids, :, j % 16].view(bits)), f"rows of sequence {s}"
    lse_plain = torch.empty(len(rows), H, device="cuda")
    O_plain, _ = B.attn_prompt(p, q_plain, *plain, table, at, new_len, lse=lse_plain)
    # both are within the bound of the exact result, which is at most (|plain| + TOL rms) / (1 - TOL): 2.1 where 2 (1 + 2 TOL) is 2.08
    ref = O_plain.double()
    off = (O[rows].double() - ref).abs() - 2.1 * TOL[dtype] * (ref.abs() + ref.pow(2).mean().sqrt())
    assert float(off.max()) <= 0 and torch.allclose(lse[rows], lse_plain, atol=2e-4, rtol=2e-4)


# ---- long and wide calls ----


@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("window", [0, 3000])
def test_row_tiles_of_many_heads_over_long_histories(dtype, d, window):
    new = [64, 0, 33, 64]
    c = TreeCache([64 + 6000, 40, 33 + 2500, 64 + 9], 16, 2, d, 32, dtype, new=new, window=window, seed=d)
    Q, O, lse = run_tree(c, strided=True)
    check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128), ("bf16", 32)])
def test_one_long_history_among_many_short_ones(dtype, d):
    rng = np.random.default_rng(1)
    new = [int(x) for x in rng.integers(0, 30, 90)]
    kv = [n + int(rng.integers(0, 40)) for n in new]
    new[70], kv[70] = 25, 8000
    c = TreeCache(kv, 4, 2, d, 16, dtype, new=new, seed=2, max_pages=500)
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)
    _, O2, lse2 = run_tree(c, Q=Q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("S,N,page,width", [(1500, 2050, 8, 6), (3, 1100, 16, 40), (1100, 2, 16, 9)])
def test_fork_of_many_sequences(S, N, page, width):
    table, lens, refs, rng = state(S, page, width, 2 * (S + N) * width, N)
    run_fork(table, lens, refs, [int(x) for x in rng.integers(-1, S, N)], page, 3)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("w,k,v", [(64, 64, 20000), (20, 64, 30000), (5, 50, 60000), (64, 1, 9001), (1, 64, 100001)])
def test_many_beams_with_rows_in_several_runs(dtype, w, k, v):
    logits, score = inputs(1, w, v, dtype, v)
    run_beam(logits, score, k)
    logits[0, w // 2] += 8.0  # (its log-probabilities stay)
    logits[0, 0, v // 2:] = float("-inf")
    score[0, w - 1] = float("-inf")
    run_beam(logits, score * 0.01, k)
    run_beam(torch.zeros(1, w, v, dtype=DTYPES[dtype]), torch.zeros(1, w), k)


# ---- offsets, streams, graphs, memory ----


@pytest.mark.parametrize("dtype,new", [("bf16", [40, 9]), ("bf16", [1, 2]), ("fp32", [40, 9]), ("fp32", [1, 1])])
def test_offsets_beyond_32_bits(dtype, new):
    d, G, page, n_pages = 128, 8, 64, 33000
    assert n_pages * G * page * d > 2**31
    c = TreeCache([150, 70], 16, G, d, page, dtype, new=new, seed=7)
    Kc, Vc, _, cu, kv_len = c.dev()
    big = [torch.zeros(n_pages, G, page, d, dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    home = {int(i): n_pages - 1 - 2 * k for k, i in enumerate(np.unique(c.table[c.table >= 0])) if i < c.p.n_pages}
    for i, to in home.items():
        big[0][to], big[1][to] = Kc[i], Vc[i]
    table = torch.tensor([[home.get(int(i), -1) for i in row] for row in c.table[:, 0]], dtype=torch.int32).cuda()
    p = B.PagedParams(**{**c.p.__dict__, "n_pages": n_pages})
    Q, lse = c.normal(c.T, 16, d), torch.empty(c.T, 16, device="cuda")
    O, _ = B.attn_tree(p, Q.cuda(), *big, table, cu, kv_len, c.mask(), lse=lse)
    check(O, lse, *c.want_tree(Q), dtype)
    turn = [x.cuda() for x in rope(p.capacity, d)]
    k, v = c.normal(c.T, G, d), c.normal(c.T, G, d)
    B.kv_append_tree(p, k.cuda(), v.cuda(), *big, table, cu, kv_len, c.mask(), rope=turn)
    last = int(table[0, 2])
    assert torch.equal(big[1][last, :, 149 % page].cpu(), v[new[0] - 1])
    B.kv_accept(p, i32([[new[0] - 1], [0]]), *big, table, cu, kv_len)
    to = 150 - new[0]
    assert torch.equal(big[1][int(table[0, to // page]), :, to % page].cpu(), v[new[0] - 1])
    B.kv_copy_pages(p, i32([[last, 1, page], [last, n_pages - 2, 3]]), *big)
    for b in big:
        bits = torch.int32 if dtype == "fp32" else torch.int16
        assert torch.equal(b[1].view(bits), b[last].view(bits))
        assert torch.equal(b[n_pages - 2, :, :3].view(bits), b[last, :, :3].view(bits)) and not b[n_pages - 2, :, 3:].any()
        for to in [*home.values(), 1, n_pages - 2]:
            b[to] = 0
        assert not b.any(), "a page that nobody names was written"


@pytest.mark.parametrize("dtype,d,new", [("bf16", 64, [30, 17, 64]), ("bf16", 128, [1, 2, 1]), ("fp32", 32, [20, 1, 3])])
def test_trees_on_other_streams_and_in_graphs(dtype, d, new):
    c = TreeCache([5000, 80, 400], 8, 2, d, 16, dtype, seed=5, new=new)
    Kc, Vc, table, cu, kv_len = c.dev()
    q, k, v = (c.normal(c.T, n, d).cuda() for n in (8, 2, 2))
    mask, turn = c.mask(), [x.cuda() for x in rope(c.cap, d)]
    O, q_rot, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(c.T, 8, device="cuda")
    keep, new_len = i32([[n - 1] for n in new]), torch.empty(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, B.paged_workspace_bytes(c.p, B.WS_TREE)), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        B.kv_append_tree(c.p, k, v, Kc, Vc, table, cu, kv_len, mask, Q=q, rope=turn, Q_rot=q_rot, stream=stream)
        B.attn_tree(c.p, q_rot, Kc, Vc, table, cu, kv_len, mask, O=O, lse=lse, ws=ws, stream=stream)
        B.kv_accept(c.p, keep, Kc, Vc, table, cu, kv_len, new_len=new_len, stream=stream)

    def result():
        torch.cuda.synchronize()
        bits = torch.int32 if dtype == "fp32" else torch.int16
        got = [O.clone(), lse.clone(), new_len.clone(), Kc.view(bits).clone(), Vc.view(bits).clone()]
        for x in (O, lse, new_len):
            x.zero_()
        ws.fill_(255)
        return got

    def same(a, b):
        assert all(torch.equal(x, y) for x, y in zip(a, b))

    step()
    eager = result()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    same(result(), eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        q.copy_(c.normal(c.T, 8, d))
        k.copy_(c.normal(c.T, 2, d))
        mask.copy_(torch.tensor([signed(int(x)) for x in c.rng.integers(0, 2**63, c.T)]))
        kv_len.copy_(i32([5000 - 900 * i, 80 - i, 400 - i]))
        graph.replay()
        got = result()
        step()
        same(result(), got)


def test_forks_and_beams_on_other_streams_and_in_graphs():
    for S, N, n_pages in ((12, 20, 900), (90, 200, 9000)):  # (one workgroup, several launches)
        table, lens, refs, rng = state(S, 8, 20, n_pages, 3)
        p = B.PagedParams(S=S, T=1, H=2, G=2, d=32, page=8, n_pages=n_pages, max_pages=20)
        table, lens, refs = i32(table), i32(lens), i32(refs)
        pristine = [torch.randn(n_pages, 2, 8, 32, device="cuda") for _ in range(2)]
        caches = [torch.empty_like(x) for x in pristine]
        w, v = 4, 3001
        bp = B.BeamParams(B=N // 4, W=w, K=4, V=v, dtype=B.F32)
        logits, score = torch.randn(N, v, device="cuda"), torch.randn(N // 4, w, device="cuda")
        parent, token = (torch.empty(N // 4, 4, dtype=torch.int32, device="cuda") for _ in range(2))
        out_score, out_ended = torch.empty(N // 4, 4, device="cuda"), torch.empty(N // 4, 4, dtype=torch.bool, device="cuda")
        new = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((N, 20), (N,), (n_pages,), (N, 3), (1,))]
        ws = [torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in (B.beam_workspace_bytes(bp), B.fork_workspace_bytes(p, N))]

        def step(stream=None):
            B.beam_select(bp, logits, score, parent=parent, token=token, out_score=out_score, out_ended=out_ended, ws=ws[0], stream=stream)
            B.kv_fork(p, parent.view(-1), table, lens, refs, grow=9, new_table=new[0], new_len=new[1], new_refs=new[2], copies=new[3],
                      missing=new[4], ws=ws[1], stream=stream)
            B.kv_copy_pages(p, new[3], *caches, stream=stream)

        def result():
            torch.cuda.synchronize()
            got = [x.clone() for x in (parent, token, out_score, *new, *caches)]
            for x in (parent, token, out_score, *new):
                x.zero_()
            for x in ws:
                x.fill_(255)
            for x, was in zip(caches, pristine):
                x.copy_(was)
            torch.cuda.synchronize()
            return got

        result()
        step()
        eager = result()
        side = torch.cuda.Stream()
        step(side)
        assert all(torch.equal(x, y) for x, y in zip(result(), eager))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(4):
            logits.copy_(torch.randn(N, v))
            lens.copy_(i32([int(x) for x in rng.integers(0, 161, S)]))
            graph.replay()
            got = result()
            step()
            assert all(torch.equal(x, y) for x, y in zip(result(), got)), f"replay {i}"


def calls(c, Kc, Vc, table, cu, kv_len, q, k, v, turn, stream=None):
    """Every call with what it allocates itself, then with outputs that are given: its results."""
    mask = c.mask()
    refs = torch.bincount(table[(table >= 0) & (table < c.p.n_pages)].long(), minlength=c.p.n_pages).int()
    bp = B.BeamParams(B=3, W=4, K=8, V=50001, dtype=B.F32)
    g = torch.Generator().manual_seed(1)
    logits, score, parent, keep = torch.randn(12, 50001, generator=g).cuda(), torch.randn(3, 4, generator=g).cuda(), i32([2, 1, 1, 1]), i32([[3], [0], [1]])
    torch.cuda.synchronize()
    q_rot = B.kv_append_tree(c.p, k, v, Kc, Vc, table, cu, kv_len, mask, Q=q, rope=turn, stream=stream)
    O, _ = B.attn_tree(c.p, q_rot, Kc, Vc, table, cu, kv_len, mask, stream=stream)
    new_len = B.kv_accept(c.p, keep, Kc, Vc, table, cu, kv_len, stream=stream)
    fork = B.kv_fork(c.p, parent, table, kv_len, refs, grow=1, stream=stream)
    beam = B.beam_select(bp, logits, score, stream=stream)
    got = [q_rot, O, new_len, *fork, *beam]
    to = [torch.zeros_like(x) for x in got]
    torch.cuda.synchronize()
    B.kv_append_tree(c.p, k, v, Kc, Vc, table, cu, kv_len, mask, Q=q, rope=turn, Q_rot=to[0], stream=stream)
    B.attn_tree(c.p, to[0], Kc, Vc, table, cu, kv_len, mask, O=to[1], stream=stream)
    B.kv_accept(c.p, keep, Kc, Vc, table, cu, kv_len, new_len=to[2], stream=stream)
    B.kv_fork(c.p, parent, table, kv_len, refs, grow=1, new_table=to[3], new_len=to[4], new_refs=to[5], copies=to[6], missing=to[7], stream=stream)
    B.beam_select(bp, logits, score, parent=to[8], token=to[9], out_score=to[10], out_ended=to[11], stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, to))
    return got


def given():
    c = TreeCache([3000, 17, 400], 8, 2, 64, 16, "bf16", seed=5, new=[9, 4, 30])
    q, k, v = (c.normal(c.T, n, 64).cuda() for n in (8, 2, 2))
    return c, (*c.dev(), q, k, v, [x.cuda() for x in rope(c.cap, 64)])


def test_buffers_of_a_call_belong_to_its_stream(monkeypatch):
    c, args = given()
    want = calls(c, *args)
    empty, on = torch.empty, []

    def noted(*a, **kw):
        on.append(torch.cuda.current_stream())
        return empty(*a, **kw)

    side = torch.cuda.Stream()
    monkeypatch.setattr(torch, "empty", noted)
    got = calls(c, *args, stream=side)
    monkeypatch.undo()
    assert len(on) >= 9 and all(s == side for s in on)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_python_path_gives_the_same(monkeypatch):
    c, args = given()
    want = calls(c, *args)
    monkeypatch.setattr(B, "_fast", B.PYTHON_PATH)
    assert all(torch.equal(a, b) for a, b in zip(calls(c, *args), want))
