"""Drafted trees over the paged cache against their definitions in 64 bits: attention, the append by tree positions, the accepted path."""
import numpy as np
import pytest
import torch

from paged_util import DTYPES, LSE_TOL, TOL, check, guarded
from paper_2512_13368_amd import binding as B
from test_gpu_paged import rope, rotated
from tree_util import TreeCache, tree_masks

pytestmark = pytest.mark.gpu


def run_tree(c, Q=None, strided=False, stream=None, ws=None):
    Kc, Vc, table, cu, kv_len = c.dev()
    Q = c.normal(c.T, c.H, c.d) if Q is None else Q
    if strided:
        wide = torch.full((c.T, (c.H + 2) * c.d), float("nan"), dtype=Q.dtype)
        wide[:, c.d:-c.d] = Q.reshape(c.T, -1)
        dq = wide.cuda()[:, c.d:-c.d].unflatten(1, (c.H, c.d))
    else:
        dq = Q.cuda()
    O, clean = guarded(c.T, c.H, c.d, c.dtype)
    lse = torch.empty(c.T, c.H, device="cuda")
    print(f"tree {c.p} new={c.new} kv_len={c.kv_len}", flush=True)
    B.attn_tree(c.p, dq, Kc, Vc, table, cu, kv_len, c.mask(), O=O, lse=lse, ws=ws, stream=stream)
    torch.cuda.synchronize()
    assert clean(), "rows behind the output were written"
    return Q, O, lse


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,page", [(8, 8), (16, 16), (32, 32), (64, 64), (128, 16), (128, 8), (64, 256)])
def test_tree_lengths(dtype, d, page):
    new = [1, 0, 5, 16, 17, 33, 64, 0, 7, 64]
    past = [0, 0, 3, 31, 100, 64, 190, 5, 1, 0]
    c = TreeCache([n + b for n, b in zip(new, past)], 4, 2, d, page, dtype, new=new, seed=d + page)
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (6, 2), (16, 1), (40, 1), (8, 8)])
def test_tree_head_layouts(dtype, H, G):
    c = TreeCache([150, 9, 70], H, G, 64, 16, dtype, new=[20, 9, 3], seed=H)
    Q, O, lse = run_tree(c, strided=True)
    check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128), ("bf16", 16)])
@pytest.mark.parametrize("window", [1, 3, 40, 129, 5000])
def test_tree_window(dtype, d, window):
    c = TreeCache([400, 33, 1, 0, 257], 4, 2, d, 16, dtype, new=[40, 7, 1, 0, 64], window=window, seed=window)
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("bf16", 64), ("bf16", 128), ("fp32", 8)])
def test_tree_masks_of_any_kind(dtype, d):
    # nothing; everything; later tokens alone; not itself; bits behind the tree; a path; all bits set
    n = 9
    odd = [0, (1 << n) - 1, 0b111110000, ((1 << n) - 1) & ~(1 << 3), 1 << 40 | 1 << 63, 0b101010101, (1 << 64) - 1, 1 << 8, 0]
    full = tree_masks(list(range(-1, 63)))
    c = TreeCache([n, 200, 64, 2], 6, 2, d, 16, dtype, new=[n, n, 64, 2], masks=[odd, odd, full, [0, 0]], seed=3)
    Q, O, lse = run_tree(c)
    want = c.want_tree(Q)
    assert torch.isinf(want[1][0]).all() and torch.isinf(want[1][-2:]).all()  # rows that see nothing
    check(O, lse, *want, dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_tree_of_a_path_is_a_prompt(dtype, d):
    new, kv = [3, 40, 64, 1], [300, 41, 513, 260]
    c = TreeCache(kv, 8, 2, d, 16, dtype, new=new, masks=[tree_masks(list(range(-1, n - 1))) for n in new], window=100, seed=4)
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_tree_of_more_than_64_tokens(dtype, d):
    # tokens from the 65th on see what their masks name of the first 64, and are seen by none
    n = 100
    masks = tree_masks([i // 2 - 1 for i in range(64)]) + [(1 << (i % 64)) | 1 for i in range(64, n)]
    c = TreeCache([n + 50, 30], 4, 2, d, 16, dtype, new=[n, 5], masks=[masks, tree_masks([-1, 0, 0, 1, 2])], seed=4)
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype,d,H", [("fp32", 32, 2), ("bf16", 64, 2), ("bf16", 128, 2), ("bf16", 32, 1)])
def test_tree_windows_of_tokens_that_see_64_others(dtype, d, H):
    # (the 65th and later stand 64 positions behind the history, one more than any of the first 64 can)
    for window in range(80, 80 + 33):
        c = TreeCache([66 + 200, 3], H, 1, d, 16, dtype, new=[66, 1], masks=[[(1 << 64) - 1] * 66, [1]], window=window, seed=4)
        if window % 8 == 0:
            Q, O, lse = run_tree(c)
            check(O, lse, *c.want_tree(Q), dtype)
            continue
        Q = c.normal(c.T, H, d)
        _, O, lse = run_tree(c, Q=Q)
        for t in (0, 63, 64, 65):
            for h in range(H):
                o, x = c.attend_tree(Q[t, h], 0, t, h)
                assert float((O[t, h].double().cpu() - o).abs().max()) <= 2 * TOL[dtype] * float(o.pow(2).mean().sqrt() + o.abs().max())
                assert abs(float(lse[t, h]) - x) <= LSE_TOL * (1 + abs(x)), f"window {window} token {t}"


@pytest.mark.parametrize("dtype,d,past", [("fp32", 64, 9000), ("bf16", 64, 20011), ("bf16", 128, 30000), ("fp32", 128, 5000), ("bf16", 8, 12000)])
def test_tree_long_histories_split_and_joined(dtype, d, past):
    c = TreeCache([past, 77, 0, past // 3], 4, 2, d, 32, dtype, new=[21, 30, 0, 1], seed=5)
    assert B.paged_workspace_bytes(c.p, B.WS_TREE) > 0
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)
    _, O2, lse2 = run_tree(c, Q=Q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2), "two calls on the same inputs differ"


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_tree_capacity_and_short_lengths(dtype, d):
    # slots beyond the capacity, before position 0, and lengths below 0
    c = TreeCache([48, 64, 50, 3], 2, 1, d, 16, dtype, new=[20, 30, 20, 3], max_len=50, seed=9)
    c.kv_len = [60, 64, -7, 1]
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)
    # (the largest lengths: all of the history, or nothing)
    c = TreeCache([50] * 4, 2, 1, d, 16, dtype, new=[20, 30, 20, 3], max_len=50, seed=9)
    c.kv_len = [2**31 - 1, 2**31 - 30, 2**31 - 1, 50]
    for window in (0, 5, 2**31 - 2):
        c.window = c.p.window = window
        Q, O, lse = run_tree(c)
        check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,page", [(32, 8), (64, 16), (128, 64)])
def test_tree_pages_out_of_range_are_masked(dtype, d, page):
    c = TreeCache([200, 150, page], 4, 2, d, page, dtype, seed=page, new=[40, 7, 1])
    c.table[0, 0, 1], c.table[1, 0, 0], c.table[2, 0, 0] = -1, c.p.n_pages, 2**31 - 1
    c.table[0, 0, 199 // page] = -5  # drafted tokens without a page
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_tree_rows_that_no_sequence_owns_stay(dtype, d):
    c = TreeCache([4000, 9], 4, 2, d, 16, dtype, new=[40, 9], seed=9)
    c.T += 70
    c.p.T = c.T
    Kc, Vc, table, cu, kv_len = c.dev()
    Q = c.normal(c.T, 4, d)
    O = torch.full((c.T, 4, d), 5.0, dtype=DTYPES[dtype], device="cuda")
    lse = torch.full((c.T, 4), 5.0, device="cuda")
    B.attn_tree(c.p, Q.cuda(), Kc, Vc, table, cu, kv_len, c.mask(), O=O, lse=lse)
    torch.cuda.synchronize()
    assert (O[49:] == 5.0).all() and (lse[49:] == 5.0).all()
    wO, wl = c.want_tree(Q[:49])
    check(O[:49], lse[:49], wO, wl, dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_tree_many_sequences(dtype, d):
    rng = np.random.default_rng(3)
    new = [int(x) for x in rng.integers(0, 20, 150)]
    c = TreeCache([n + int(rng.integers(0, 300)) for n in new], 2, 2, d, 8, dtype, new=new, seed=6)
    Q, O, lse = run_tree(c)
    check(O, lse, *c.want_tree(Q), dtype)


def run_append(c, with_q=True, with_rope=True):
    Kc, Vc, table, cu, kv_len = c.dev()
    T, H, G, d = c.T, c.H, c.G, c.d
    qkv = c.normal(T, (H + 2 * G) * d)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([H * d, G * d, G * d], 1))
    dq, dk, dv = (x.unflatten(1, (-1, d)) for x in qkv.cuda().split([H * d, G * d, G * d], 1))
    cos, sin = rope(c.cap, d)
    Q_rot, clean = guarded(T, H, d, c.dtype)
    print(f"append {c.p} new={c.new} kv_len={c.kv_len}", flush=True)
    B.kv_append_tree(c.p, dk, dv, Kc, Vc, table, cu, kv_len, c.mask(), Q=dq if with_q else None,
                     rope=(cos.cuda(), sin.cuda()) if with_rope else None, Q_rot=Q_rot if with_q else None)
    torch.cuda.synchronize()
    assert clean()
    half = 2.0 ** -8 if c.dtype == "bf16" else 2.0 ** -22  # half a unit of the type; of fp32, of the two roundings on the way
    mine = torch.zeros(c.K_cache.shape[:3], dtype=torch.bool)
    for s, n in enumerate(c.new):
        for i in range(n):
            t, slot = int(c.cu[s]) + i, max(c.kv_len[s], 0) - n + i
            pos = c.sees(s, i)[0]
            here = 0 <= slot < c.cap and 0 <= pos < c.cap
            if with_q:
                want = rotated(q[t], cos[pos], sin[pos]) if here else torch.zeros(H, d)
                assert float(((Q_rot[t].double().cpu() - want).abs() - 2e-7 * 4 - want.abs() * half).max()) <= 0
            page = int(c.table[s, 0, slot // c.page]) if here else -1
            if not 0 <= page < c.p.n_pages:
                continue
            mine[page, :, slot % c.page] = True
            assert torch.equal(Vc[page, :, slot % c.page].cpu(), v[t])
            got, want = Kc[page, :, slot % c.page].cpu(), rotated(k[t], cos[pos], sin[pos])
            if with_rope:
                assert float(((got.double() - want).abs() - 2e-7 * 4 - want.abs() * half).max()) <= 0
            else:
                assert torch.equal(got, k[t])
    bits = torch.int32 if c.dtype == "fp32" else torch.int16
    for got, was in ((Kc, c.K_cache), (Vc, c.V_cache)):
        assert torch.equal(got.cpu().view(bits)[~mine], was.view(bits)[~mine]), "rows of other positions changed"


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,G,d,page", [(2, 2, 8, 8), (4, 1, 16, 16), (3, 3, 32, 64), (6, 2, 64, 16), (32, 8, 128, 256)])
def test_append_by_tree_positions(dtype, H, G, d, page):
    run_append(TreeCache([1, 0, 20, 64, 100], H, G, d, page, dtype, new=[1, 0, 20, 3, 64], seed=d))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_append_tree_without_queries_without_rotation_and_without_a_place(dtype):
    c = TreeCache([40, 3], 4, 2, 32, 16, dtype, new=[40, 2], seed=1)
    run_append(c, with_q=False)
    run_append(c, with_q=False, with_rope=False)
    c = TreeCache([48, 64, 30, 70], 4, 2, 32, 16, dtype, new=[40, 30, 20, 70], max_len=50, seed=9)
    c.kv_len = [60, 64, -7, 70]
    c.table[0, 0, 1] = -1
    run_append(c)


def run_accept(c, keep, width=None):
    Kc, Vc, table, cu, kv_len = c.dev()
    width = width or max(len(k) for k in keep)
    rows = torch.tensor([(k + [-1] * width)[:width] for k in keep], dtype=torch.int32)
    print(f"accept {c.p} keep={keep}", flush=True)
    new_len = B.kv_accept(c.p, rows.cuda(), Kc, Vc, table, cu, kv_len)
    torch.cuda.synchronize()
    want_k, want_v = c.K_cache.clone(), c.V_cache.clone()
    for s, n in enumerate(c.new):
        past, m = max(c.kv_len[s], 0) - n, 0
        for i, k in enumerate(rows[s].tolist()):
            if not (0 <= k < n and (i == 0 or k > rows[s, i - 1])):
                break
            m += 1
            src, dst = past + k, past + i
            if not (0 <= dst and src < c.cap):
                continue
            a, b = int(c.table[s, 0, src // c.page]), int(c.table[s, 0, dst // c.page])
            if 0 <= a < c.p.n_pages and 0 <= b < c.p.n_pages:
                want_k[b, :, dst % c.page], want_v[b, :, dst % c.page] = c.K_cache[a, :, src % c.page], c.V_cache[a, :, src % c.page]
        assert int(new_len[s]) == past + m
    bits = torch.int32 if c.dtype == "fp32" else torch.int16
    assert torch.equal(Kc.cpu().view(bits), want_k.view(bits)) and torch.equal(Vc.cpu().view(bits), want_v.view(bits))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("G,d,page", [(1, 8, 8), (2, 32, 16), (8, 128, 16), (3, 64, 128), (5, 128, 32)])
def test_accepted_path_follows_the_history(dtype, G, d, page):
    c = TreeCache([30, 64, 70, 9, 100], G, G, d, page, dtype, new=[20, 64, 1, 9, 64], seed=d)
    run_accept(c, [[1, 2, 7, 19], list(range(1, 64)), [0], [], [0, 1, 2, 30, 31, 62, 63]])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_accepted_lists_that_end_early_and_rows_without_a_place(dtype):
    # a list ends where it does not ascend, is below 0, or names no drafted token; then more entries than 64, and trees beyond 64 tokens
    c = TreeCache([30, 30, 30, 30], 2, 2, 32, 8, dtype, new=[10, 10, 10, 0], seed=2)
    run_accept(c, [[3, 3, 4], [2, -1, 5], [9, 10, 11], [0, 1]])
    c = TreeCache([150, 300], 2, 2, 32, 8, dtype, new=[130, 200], seed=2)
    run_accept(c, [list(range(1, 130)), [*range(0, 70), *range(90, 200)]])
    c = TreeCache([48, 64, 30], 2, 2, 32, 16, dtype, new=[20, 30, 20], max_len=50, seed=9)
    c.kv_len = [60, 64, -7]
    c.table[0, 0, 2] = -1
    run_accept(c, [[2, 5, 19], [10, 11, 20], [1, 2]])
