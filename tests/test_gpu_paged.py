"""The paged cache's operators against their definitions in 64 bits: lengths, head layouts, pages, windows, types, empty rows,
rows and entries that may hold anything, strides, streams, graphs."""
import numpy as np
import pytest
import torch

from paged_util import DTYPES, Cache, check, guarded
from paper_2512_13368_amd import binding as B

pytestmark = pytest.mark.gpu

LENGTHS = [1, 0, 7, 8, 9, 31, 32, 33, 64, 65, 127, 300]


def run_decode(c, Q=None, strided=False, stream=None, ws=None):
    Kc, Vc, table, _, kv_len = c.dev()
    S = len(c.kv_len)
    Q = c.normal(S, c.H, c.d) if Q is None else Q
    if strided:
        wide = torch.full((S, (c.H + 2) * c.d), float("nan"), dtype=Q.dtype)
        wide[:, c.d:-c.d] = Q.reshape(S, -1)
        dq = wide.cuda()[:, c.d:-c.d].unflatten(1, (c.H, c.d))
    else:
        dq = Q.cuda()
    O, clean = guarded(S, c.H, c.d, c.dtype)
    lse = torch.empty(S, c.H, device="cuda")
    print(f"decode {c.p}", flush=True)
    B.attn_decode(c.p, dq, Kc, Vc, table, kv_len, O=O, lse=lse, ws=ws, stream=stream)
    torch.cuda.synchronize()
    assert clean(), "rows behind the output were written"
    return Q, O, lse


def run_prompt(c, Q=None, strided=False):
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
    print(f"prompt {c.p} new={c.new} kv_len={c.kv_len}", flush=True)
    B.attn_prompt(c.p, dq, Kc, Vc, table, cu, kv_len, O=O, lse=lse)
    torch.cuda.synchronize()
    assert clean(), "rows behind the output were written"
    return Q, O, lse


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,page", [(8, 8), (16, 16), (32, 32), (64, 64), (128, 16), (128, 8), (64, 256)])
def test_decode_lengths(dtype, d, page):
    c = Cache(LENGTHS, 4, 2, d, page, dtype, seed=d + page)
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (6, 2), (16, 1), (17, 1), (40, 1), (8, 8)])
def test_decode_head_layouts(dtype, H, G):
    c = Cache([130, 5, 0, 64], H, G, 64, 16, dtype, seed=H)
    Q, O, lse = run_decode(c, strided=True)
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("window", [1, 8, 33, 5000])
def test_decode_window(dtype, window):
    c = Cache([400, 33, 1, 0, 257], 4, 2, 32, 16, dtype, window=window, seed=window)
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_decode_one_long_sequence_split_and_joined(dtype):
    c = Cache([20011], 4, 2, 64, 32, dtype, seed=5)
    assert B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)
    _, O2, lse2 = run_decode(c, Q=Q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2), "two calls on the same inputs differ"


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_decode_pages_listed_per_head(dtype):
    c = Cache([100, 64, 1, 0], 6, 3, 64, 32, dtype, per_head=True, seed=8)
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_decode_wide_tables_and_capacity(dtype):
    # a table far wider than the sequences need (split for lengths that none has), then lengths beyond what may be held
    c = Cache([40, 700, 3], 2, 1, 64, 16, dtype, max_pages=4096, seed=2, spare=0)
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)
    for over in (dict(max_pages=3), dict(max_len=37), dict(max_len=37, window=20)):
        c = Cache([48, 30, 39], 2, 1, 32, 16, dtype, seed=3, **over)
        c.kv_len = [60, 30, -4]
        Q, O, lse = run_decode(c)
        check(O, lse, *c.want_decode(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("page", [8, 16, 64])
def test_pages_out_of_range_are_masked(dtype, page):
    c = Cache([200, 150, page], 4, 2, 32, page, dtype, seed=page, new=[40, 7, 1])
    c.table[0, 0, 1], c.table[1, 0, 0], c.table[2, 0, 0] = -1, c.p.n_pages, 2**31 - 1
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("op", ["decode", "prompt"])
def test_logits_of_any_size_and_minus_infinity(op):
    # logits up to +-3e4, and one key of a sequence whose logits are -inf: no weight; another of nothing else: as if it saw none
    c = Cache([90, 33], 2, 1, 32, 8, "fp32", seed=4, new=[30, 33])
    ids = c.table[0, 0].astype(np.int64)
    c.K_cache[ids[0], 0, 3] = float("-inf")
    c.K_cache[ids[5], 0] *= 1000.0
    for i in c.table[1, 0][:-(-33 // 8)]:
        c.K_cache[int(i)] = float("-inf")
    Q = c.normal(2 if op == "decode" else c.T, 2, 32).abs() + 0.01
    run, want = (run_decode, c.want_decode) if op == "decode" else (run_prompt, c.want_prompt)
    Q, O, lse = run(c, Q=Q)
    wO, wl = want(Q)
    last = 1 if op == "decode" else 30
    wO[last:], wl[last:] = 0.0, float("-inf")
    assert torch.equal(O[last:].double().cpu(), wO[last:]) and torch.equal(lse[last:].double().cpu(), wl[last:])
    # (logits of 3e4 are off by their own rounding, 3e4 * 32 * 2^-24 = 0.06 at most: the weights by that, relatively)
    assert torch.isfinite(O).all() and float((O[:last].double().cpu() - wO[:last]).abs().max()) <= 0.13 * float(wO.abs().max())
    assert float((lse[:last].double().cpu() - wl[:last]).abs().max()) <= 0.13


def test_nan_stays_with_its_sequence_and_key_head():
    c = Cache([90, 33, 70], 4, 2, 64, 16, "bf16", seed=4, new=[9, 33, 1])
    c.V_cache[int(c.table[1, 0, 1]), 1, 2] = float("nan")
    for run in (run_decode, run_prompt):
        _, O, _ = run(c)
        O = O.cpu()
        rows = slice(1, 2) if run is run_decode else slice(9, 42)
        bad = torch.isnan(O).any(-1)
        assert bad[rows, 2:][-1].all(), "a NaN that a query sees comes out"
        bad[rows, 2:] = False
        assert not bad.any(), "and reaches no other sequence and no other key head's queries"


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,page", [(8, 8), (16, 16), (32, 32), (64, 16), (128, 64), (128, 8), (64, 256)])
def test_prompt_packed_lengths(dtype, d, page):
    new = [1, 0, 5, 16, 17, 33, 130, 0, 64]
    c = Cache(new, 4, 2, d, page, dtype, new=new, seed=d + page)
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("window", [0, 1, 40, 129])
def test_prompt_chunks_over_a_past(dtype, d, window):
    new, kv = [3, 70, 1, 200], [300, 71, 513, 260]
    c = Cache(kv, 3, 1, d, 16, dtype, new=new, window=window, seed=window)
    Q, O, lse = run_prompt(c, strided=True)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,G", [(1, 1), (5, 1), (12, 4), (16, 1), (24, 1), (8, 8)])
def test_prompt_head_layouts(dtype, H, G):
    c = Cache([130, 9, 40], H, G, 64, 32, dtype, new=[130, 2, 40], seed=H)
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_prompt_many_sequences(dtype, d):
    new = [int(x) for x in np.random.default_rng(3).integers(0, 40, 150)]
    c = Cache([n + 3 * (i % 5) for i, n in enumerate(new)], 2, 2, d, 8, dtype, new=new, seed=6)
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_prompt_more_new_tokens_than_positions_and_beyond_the_capacity(dtype, d):
    # tokens before position 0 see nothing; those beyond the capacity see what is held
    c = Cache([40, 64, 50], 4, 2, d, 16, dtype, new=[48, 30, 20], max_len=60, seed=9)
    c.kv_len = [40, 64, -7]
    Q, O, lse = run_prompt(c)
    wO, wl = c.want_prompt(Q)
    assert torch.isinf(wl[:8]).all() and torch.isinf(wl[78:]).all()
    check(O, lse, wO, wl, dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_prompt_rows_that_no_sequence_owns_stay(dtype, d):
    c = Cache([40, 9], 4, 2, d, 16, dtype, new=[40, 9], seed=9)
    c.T += 200
    c.p.T = c.T
    Kc, Vc, table, cu, kv_len = c.dev()
    Q = c.normal(c.T, 4, d)
    O = torch.full((c.T, 4, d), 5.0, dtype=DTYPES[dtype], device="cuda")
    lse = torch.full((c.T, 4), 5.0, device="cuda")
    B.attn_prompt(c.p, Q.cuda(), Kc, Vc, table, cu, kv_len, O=O, lse=lse)
    torch.cuda.synchronize()
    assert (O[49:] == 5.0).all() and (lse[49:] == 5.0).all()
    wO, wl = c.want_prompt(Q[:49])
    check(O[:49], lse[:49], wO, wl, dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("bf16", 64), ("bf16", 128)])
def test_prompt_of_one_token_is_decode(dtype, d):
    kv = [1, 77, 300, 32]
    c = Cache(kv, 8, 2, d, 16, dtype, seed=1)
    Q, O, lse = run_decode(c)
    _, O2, lse2 = run_prompt(c, Q=Q)
    wO, wl = c.want_decode(Q)
    check(O, lse, wO, wl, dtype)
    check(O2, lse2, wO, wl, dtype)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_prompt_of_a_few_tokens_over_a_long_past(dtype, d):
    c = Cache([9001, 12345], 4, 2, d, 32, dtype, new=[3, 1], seed=12)
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


def rope(cap, d):
    a = np.arange(cap)[:, None] * 10000.0 ** (-2.0 * np.arange(d // 2) / d)
    return torch.from_numpy(np.cos(a)).float(), torch.from_numpy(np.sin(a)).float()


def rotated(x, cos, sin):
    z = torch.view_as_complex(x.double().reshape(*x.shape[:-1], -1, 2).contiguous()) * torch.complex(cos.double(), sin.double())
    return torch.view_as_real(z).flatten(-2)


def run_append(c, with_q=True, with_rope=True, fused=True):
    Kc, Vc, table, cu, kv_len = c.dev()
    T, H, G, d = c.T, c.H, c.G, c.d
    qkv = c.normal(T, (H + 2 * G) * d)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([H * d, G * d, G * d], 1))
    dq, dk, dv = (x.unflatten(1, (-1, d)) for x in qkv.cuda().split([H * d, G * d, G * d], 1))
    if not fused:
        dq, dk, dv = dq.contiguous(), dk.contiguous(), dv.contiguous()
    cos, sin = rope(c.cap, d)
    Q_rot, clean = guarded(T, H, d, c.dtype)
    print(f"append {c.p} new={c.new} kv_len={c.kv_len}", flush=True)
    B.kv_append(c.p, dk, dv, Kc, Vc, table, cu, kv_len, Q=dq if with_q else None, rope=(cos.cuda(), sin.cuda()) if with_rope else None,
                Q_rot=Q_rot if with_q else None)
    torch.cuda.synchronize()
    assert clean()
    # what the caches should hold: everything else as it was, to the bit
    mine = torch.zeros(c.K_cache.shape[:3], dtype=torch.bool)
    for s, n in enumerate(c.new):
        for i in range(n):
            t, pos = int(c.cu[s]) + i, c.kv_len[s] - n + i
            here = 0 <= pos < c.cap
            if with_q:
                want = rotated(q[t], cos[pos], sin[pos]) if here else torch.zeros(H, d)
                off = (Q_rot[t].double().cpu() - want).abs()
                assert float((off - 2e-7 * 4 - want.abs() * (2.0 ** -8 if c.dtype == "bf16" else 2.0 ** -22)).max()) <= 0
            page = int(c.table[s, 0, pos // c.page]) if here else -1
            if not 0 <= page < c.p.n_pages:
                continue
            mine[page, :, pos % c.page] = True
            assert torch.equal(Vc[page, :, pos % c.page].cpu(), v[t])
            got = Kc[page, :, pos % c.page].cpu()
            if with_rope:
                want = rotated(k[t], cos[pos], sin[pos])
                assert float(((got.double() - want).abs() - 2e-7 * 4 - want.abs() * (2.0 ** -8 if c.dtype == "bf16" else 2.0 ** -22)).max()) <= 0
            else:
                assert torch.equal(got, k[t])
    bits = torch.int32 if c.dtype == "fp32" else torch.int16
    for got, was in ((Kc, c.K_cache), (Vc, c.V_cache)):
        assert torch.equal(got.cpu().view(bits)[~mine], was.view(bits)[~mine]), "rows of other positions changed"


# (an entry is rounded twice in fp32 and once to the storage type: 2^-24 of values up to 4 or so twice, and half a unit of the type)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,G,d,page", [(2, 2, 8, 8), (4, 1, 16, 16), (3, 3, 32, 64), (6, 2, 64, 16), (8, 1, 128, 8), (32, 8, 128, 256)])
def test_append_places_and_rotates(dtype, H, G, d, page):
    run_append(Cache([1, 0, 20, 64, 65, 130], H, G, d, page, dtype, new=[1, 0, 20, 3, 1, 70], seed=d))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_append_one_token_each(dtype):
    run_append(Cache([5 + 3 * i for i in range(70)], 4, 2, 64, 16, dtype, seed=3), fused=False)
    run_append(Cache([33], 1, 1, 8, 8, dtype, seed=3))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_append_without_queries_and_without_rotation(dtype):
    c = Cache([40, 3], 4, 2, 32, 16, dtype, new=[40, 2], seed=1)
    run_append(c, with_q=False)
    run_append(c, with_q=False, with_rope=False)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_append_tokens_without_a_place(dtype):
    c = Cache([40, 64, 30], 4, 2, 32, 16, dtype, new=[48, 30, 20], max_len=50, seed=9)
    c.kv_len = [40, 64, -7]
    c.table[0, 0, 1] = -1
    run_append(c)


def test_offsets_beyond_32_bits():
    # caches of 2^31 elements and more: pages at both ends of them
    d, G, page, n_pages = 128, 8, 64, 33000
    assert n_pages * G * page * d > 2**31
    c = Cache([150, 70], 16, G, d, page, "bf16", new=[150, 70], seed=7)
    Kc, Vc, _, cu, kv_len = c.dev()
    big = [torch.zeros(n_pages, G, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    home = {int(i): n_pages - 1 - 2 * k for k, i in enumerate(np.unique(c.table[c.table >= 0])) if i < c.p.n_pages}
    for i, to in home.items():
        big[0][to], big[1][to] = Kc[i], Vc[i]
    table = torch.tensor([[home.get(int(i), -1) for i in row] for row in c.table[:, 0]], dtype=torch.int32).cuda()
    p = B.PagedParams(**{**c.p.__dict__, "n_pages": n_pages})
    Q = c.normal(c.T, 16, d)
    lse = torch.empty(c.T, 16, device="cuda")
    O, _ = B.attn_prompt(p, Q.cuda(), *big, table, cu, kv_len, lse=lse)
    check(O, lse, *c.want_prompt(Q), "bf16")
    Q = c.normal(2, 16, d)
    lse = torch.empty(2, 16, device="cuda")
    O, _ = B.attn_decode(p, Q.cuda(), *big, table, kv_len, lse=lse)
    check(O, lse, *c.want_decode(Q), "bf16")
    # append writes there, and nothing else
    cos, sin = rope(p.capacity, d)
    k, v = c.normal(c.T, G, d), c.normal(c.T, G, d)
    B.kv_append(p, k.cuda(), v.cuda(), *big, table, cu, kv_len, rope=(cos.cuda(), sin.cuda()))
    last = int(table[0, 2])
    assert torch.equal(big[1][last, :, 149 % page].cpu(), v[149])
    for b in big:
        for to in home.values():
            b[to] = 0
        assert not b.any(), "a page that nobody lists was written"


def test_other_streams_and_graphs():
    c = Cache([3000, 17, 400], 8, 2, 64, 16, "bf16", seed=5, new=[1, 1, 1])
    Kc, Vc, table, cu, kv_len = c.dev()
    Q = c.normal(3, 8, 64)
    dq = Q.cuda()
    O, lse = torch.empty_like(dq), torch.empty(3, 8, device="cuda")
    ws = torch.empty(max(16, B.paged_workspace_bytes(c.p, B.WS_DECODE)), dtype=torch.uint8, device="cuda")
    cos, sin = (x.cuda() for x in rope(c.cap, 64))
    new_k, new_v, Q_rot = c.normal(3, 2, 64).cuda(), c.normal(3, 2, 64).cuda(), torch.empty_like(dq)

    def step(stream=None):
        B.kv_append(c.p, new_k, new_v, Kc, Vc, table, cu, kv_len, Q=dq, rope=(cos, sin), Q_rot=Q_rot, stream=stream)
        B.attn_decode(c.p, Q_rot, Kc, Vc, table, kv_len, O=O, lse=lse, ws=ws, stream=stream)

    step()
    torch.cuda.synchronize()
    eager = O.clone(), lse.clone()
    side = torch.cuda.Stream()
    O.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert torch.equal(O, eager[0]) and torch.equal(lse, eager[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        dq.copy_(c.normal(3, 8, 64))
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone(), lse.clone()
        O.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(O, got[0]) and torch.equal(lse, got[1]), f"replay {k}"


def test_buffers_of_a_call_belong_to_its_stream(monkeypatch):
    """Memory given on to the current stream's work while a call on another still runs would be written twice."""
    c = Cache([3000, 17, 400], 8, 2, 64, 16, "bf16", seed=5, new=[1, 1, 1])
    assert B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0
    Kc, Vc, table, cu, kv_len = c.dev()
    dq = c.normal(3, 8, 64).cuda()
    cos, sin = (x.cuda() for x in rope(c.cap, 64))
    k, v = c.normal(3, 2, 64).cuda(), c.normal(3, 2, 64).cuda()
    empty, on = torch.empty, []

    def noted(*args, **kw):
        on.append(torch.cuda.current_stream())
        return empty(*args, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    monkeypatch.setattr(torch, "empty", noted)
    Q_rot = B.kv_append(c.p, k, v, Kc, Vc, table, cu, kv_len, Q=dq, rope=(cos, sin), stream=side)
    O, _ = B.attn_decode(c.p, Q_rot, Kc, Vc, table, kv_len, stream=side)
    P, _ = B.attn_prompt(c.p, Q_rot, Kc, Vc, table, cu, kv_len, stream=side)
    monkeypatch.undo()
    side.synchronize()
    assert len(on) >= 4 and all(s == side for s in on)
    again, _ = B.attn_decode(c.p, Q_rot, Kc, Vc, table, kv_len)
    assert torch.equal(O, again) and O.shape == P.shape


def test_the_python_path_gives_the_same(monkeypatch):
    c = Cache([40, 0, 9], 4, 2, 64, 16, "bf16", new=[5, 0, 9], seed=1)
    Kc, Vc, table, cu, kv_len = c.dev()
    dq = c.normal(c.T, 4, 64).cuda()
    O, lse = torch.empty_like(dq), torch.empty(c.T, 4, device="cuda")
    B.attn_prompt(c.p, dq, Kc, Vc, table, cu, kv_len, O=O, lse=lse)
    lse2 = torch.empty_like(lse)
    monkeypatch.setattr(B, "_fast", B.PYTHON_PATH)
    O2, _ = B.attn_prompt(c.p, dq, Kc, Vc, table, cu, kv_len, lse=lse2)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    cos, sin = (x.cuda() for x in rope(c.cap, 64))
    k, v = c.normal(c.T, 2, 64).cuda(), c.normal(c.T, 2, 64).cuda()
    caches = [x.clone() for x in (Kc, Vc)]
    q1 = B.kv_append(c.p, k, v, Kc, Vc, table, cu, kv_len, Q=dq, rope=(cos, sin))
    monkeypatch.undo()
    q2 = B.kv_append(c.p, k, v, *caches, table, cu, kv_len, Q=dq, rope=(cos, sin), Q_rot=torch.empty_like(dq))
    assert torch.equal(q1, q2) and torch.equal(Kc.view(torch.int16), caches[0].view(torch.int16))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,window", [(8, 0), (8, 700), (16, 0), (128, 0)])
def test_prompt_long_page_lists(d, page, window):
    # lists of more pages than a wavefront has lanes, some of them out of range, also where the list is first looked at
    c = Cache([1500, 1111], 4, 2, d, page, "bf16", new=[90, 33], window=window, seed=d + page)
    for i in {0, 3, 63, 64, 65, 127, 130, 150}:
        if i * page < 1100:
            c.table[0, 0, i], c.table[1, 0, i] = -1, c.p.n_pages + i
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), "bf16")


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_logits_that_grow_along_the_keys(d):
    # the softmax's reference has to rise many times, by a little and by a lot
    c = Cache([900], 2, 1, d, 16, "bf16", new=[200], seed=d)
    ids = c.table[0, 0].astype(np.int64)
    for j in range(900):
        c.K_cache[int(ids[j // 16]), 0, j % 16] = (j / 900.0) ** 2 * 40.0 * (1.0 if j % 7 else -1.0)
    Q = (c.normal(200, 2, d).abs() * 0.5 + 0.5).to(torch.bfloat16)
    Q, O, lse = run_prompt(c, Q=Q)
    wO, wl = c.want_prompt(Q)
    check(O, lse, wO, wl, "bf16")


# ---- the kernels of large prompt batches (128- or 64-row workgroups), on shapes small enough for the reference: sequences without
# ---- new tokens make the batch large, a wide page table makes the walks look long (keys are then split over workgroups)
CROWD = 700
TYPES = [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128), ("fp32", 32), ("bf16", 32), ("fp32", 8), ("bf16", 16), ("bf16", 8), ("fp32", 16)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page,window", [(8, 0), (32, 0), (16, 50), (64, 1)])
def test_large_batches(dtype, d, page, window):
    new = [1, 0, 5, 130, 33, 16, 64, 3]
    kv = [1, 9, 300, 130, 97, 16, 200, 70]
    c = Cache(kv + [0] * CROWD, 6, 2, d, page, dtype, new=new + [0] * CROWD, window=window, seed=d + page)
    Q, O, lse = run_prompt(c, strided=True)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("H,G", [(1, 1), (5, 1), (12, 4)])
def test_large_batches_head_layouts(dtype, d, H, G):
    c = Cache([130, 9, 40] + [0] * CROWD, H, G, d, 16, dtype, new=[130, 2, 40] + [0] * CROWD, seed=H)
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_large_batches_pages_out_of_range_and_places_outside(dtype, d):
    c = Cache([700, 150, 64] + [0] * CROWD, 4, 2, d, 8, dtype, new=[90, 60, 70] + [0] * CROWD, seed=d, max_len=650)
    c.kv_len[2] = 40  # 30 of its tokens stand before position 0
    for i in (1, 3, 63, 64, 65, 80):
        c.table[0, 0, i] = -1
    c.table[1, 0, 0], c.table[1, 0, 17] = c.p.n_pages, 2**31 - 1
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("window", [0, 333])
def test_large_walks_are_split_and_joined(dtype, d, window):
    c = Cache([2300, 0, 700, 1300], 8, 2, d, 16, dtype, new=[150, 0, 70, 1], window=window, seed=d, max_pages=40000)
    if window == 0:
        assert B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)
    _, O2, lse2 = run_prompt(c, Q=Q)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,d", [("fp32", 32), ("bf16", 64), ("bf16", 128)])
def test_split_walks_leave_rows_that_no_sequence_owns(dtype, d):
    c = Cache([400, 90], 8, 2, d, 16, dtype, new=[40, 9], seed=9, max_pages=40000)
    c.T += 300
    c.p.T = c.T
    Kc, Vc, table, cu, kv_len = c.dev()
    Q = c.normal(c.T, 8, d)
    O = torch.full((c.T, 8, d), 5.0, dtype=DTYPES[dtype], device="cuda")
    lse = torch.full((c.T, 8), 5.0, device="cuda")
    assert B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0
    B.attn_prompt(c.p, Q.cuda(), Kc, Vc, table, cu, kv_len, O=O, lse=lse)
    torch.cuda.synchronize()
    assert (O[49:] == 5.0).all() and (lse[49:] == 5.0).all()
    check(O[:49], lse[:49], *c.want_prompt(Q[:49]), dtype)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 32)])
def test_large_batches_logits_that_grow_along_the_keys(dtype, d):
    # the softmax's reference has to rise many times, by a little and by a lot
    c = Cache([900] + [0] * CROWD, 2, 1, d, 16, dtype, new=[200] + [0] * CROWD, seed=d)
    ids = c.table[0, 0].astype(np.int64)
    for j in range(900):
        c.K_cache[int(ids[j // 16]), 0, j % 16] = (j / 900.0) ** 2 * 40.0 * (1.0 if j % 7 else -1.0)
    Q = (c.normal(200, 2, d).abs() * 0.5 + 0.5).to(DTYPES[dtype])
    Q, O, lse = run_prompt(c, Q=Q)
    wO, wl = c.want_prompt(Q)
    check(O, lse, wO, wl, dtype)


def test_many_sequences_find_their_tokens():
    # more sequences than one look at 63, or 63 at 63, takes
    rng = np.random.default_rng(5)
    for S in (63, 64, 65, 127, 4032, 4100):
        new = [int(x) for x in rng.integers(0, 3, S)]
        c = Cache(new, 1, 1, 8, 8, "fp32", new=new, seed=S)
        Q, O, lse = run_prompt(c)
        check(O, lse, *c.want_prompt(Q), "fp32")
        run_append(c)


@pytest.mark.parametrize("S", [65, 130, 300])
def test_decode_parts_over_many_sequences(S):
    # ragged lengths over more sequences than a wavefront has lanes, few heads: split into parts
    kv = [int(x) for x in np.random.default_rng(S).integers(0, 3000, S)]
    kv[3], kv[64] = 0, 4000
    c = Cache(kv, 2, 1, 32, 32, "bf16", seed=S)
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), "bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_append_of_more_than_the_caches_hold(dtype):
    # written past the caches: 128 MB and more of rows; every row against the same call on a part of the tokens
    H, G, d, page = 32, 8, 128, 16
    T = 11000 if dtype == "bf16" else 5500
    n_pages = T // page + 1
    p = B.PagedParams(S=1, T=T, H=H, G=G, d=d, page=page, n_pages=n_pages, max_pages=n_pages, dtype=B.F32 if dtype == "fp32" else B.BF16)
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(DTYPES[dtype])
    q, k, v = new(T, H, d), new(T, G, d), new(T, G, d)
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)[None]
    cos, sin = (x.cuda() for x in rope(p.capacity, d))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    caches = [[torch.zeros(n_pages, G, page, d, dtype=DTYPES[dtype], device="cuda") for _ in range(2)] for _ in range(2)]
    whole = B.kv_append(p, k, v, *caches[0], table, ints(0, T), ints(T), Q=q, rope=(cos, sin))
    for lo in range(0, T, 2000):
        hi = min(T, lo + 2000)
        part = B.PagedParams(**{**p.__dict__, "T": hi - lo})
        rows = B.kv_append(part, k[lo:hi], v[lo:hi], *caches[1], table, ints(0, hi - lo), ints(hi), Q=q[lo:hi], rope=(cos, sin))
        assert torch.equal(rows, whole[lo:hi])
    assert torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])


# ---- walks of middle length: parts of a few tiles, joined by a few threads a row; the running reference of every type
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("window", [0, 1500])
def test_middle_walks_are_split_and_joined(dtype, d, window):
    c = Cache([1100, 37, 2047, 0], 6, 2, d, 16, dtype, new=[900, 37, 600, 0], window=window, seed=d + 1)
    assert B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0
    c.table[2, 0, 5] = -1
    Q, O, lse = run_prompt(c, strided=True)
    check(O, lse, *c.want_prompt(Q), dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_few_tokens_over_middle_pasts(dtype, d):
    c = Cache([1500, 40, 1030], 4, 2, d, 32, dtype, new=[10, 3, 33], seed=d + 2)
    assert B.paged_workspace_bytes(c.p, B.WS_PROMPT) > 0
    Q, O, lse = run_prompt(c)
    check(O, lse, *c.want_prompt(Q), dtype)


def growing(c, n, d):
    """Keys whose logits grow along a sequence to some 200, every seventh's sign turned."""
    ids = c.table[0, 0].astype(np.int64)
    for j in range(n):
        c.K_cache[int(ids[j // 16]), 0, j % 16] = (j / float(n)) ** 2 * 40.0 * (32 / d) ** 0.5 * (1.0 if j % 7 else -1.0)


def check_grown(O, lse, want_O, want_lse, dtype, d):
    """check(), with room for the logits' own rounding: sums of d products in 32 bits are off by d 2^-24 of a logit at most (its
    products have one sign), the weights relatively by as much, and with them numerator and denominator of an output."""
    room = 2 * d * 2.0**-24 * float(want_lse.max()) * float(want_O.abs().max())
    got = O.double().cpu()
    near = torch.where((got - want_O).abs() <= room, want_O, got - room * (got - want_O).sign())
    check(near, lse, want_O, want_lse, dtype)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("tokens", [20, 200])
def test_logits_that_grow_along_the_keys_in_every_type(dtype, d, tokens):
    c = Cache([900] + [0] * (CROWD if tokens == 200 else 0), 2, 1, d, 16, dtype, new=[tokens] + [0] * (CROWD if tokens == 200 else 0), seed=d)
    growing(c, 900, d)
    Q, O, lse = run_prompt(c, Q=(c.normal(tokens, 2, d).abs() * 0.5 + 0.5).to(DTYPES[dtype]))
    check_grown(O, lse, *c.want_prompt(Q), dtype, d)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_decode_logits_that_grow_along_the_keys(dtype, d):
    c = Cache([900], 2, 1, d, 16, dtype, seed=d)
    growing(c, 900, d)
    Q, O, lse = run_decode(c, Q=(c.normal(1, 2, d).abs() * 0.5 + 0.5).to(DTYPES[dtype]))
    check_grown(O, lse, *c.want_decode(Q), dtype, d)


@pytest.mark.parametrize("dtype,d", [("fp32", 8), ("bf16", 32), ("fp32", 128)])
def test_decode_parts_of_small_and_large_rows(dtype, d):
    c = Cache([9000, 3000], 4, 2, d, 16, dtype, seed=d)
    assert B.paged_workspace_bytes(c.p, B.WS_DECODE) > 0
    Q, O, lse = run_decode(c)
    check(O, lse, *c.want_decode(Q), dtype)
