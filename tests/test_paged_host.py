"""Refusals of the paged cache's entry points, before anything touches a GPU, and the binding's own messages."""
import ctypes

import pytest
import torch

from paper_2512_13368_amd import binding as B

vp = ctypes.c_void_p
A = vp(4096)  # fake addresses: every call must fail before they are used


def params(**kw):
    base = dict(S=2, T=6, H=4, G=2, d=64, page=16, n_pages=10, max_pages=4, dtype=B.BF16)
    base.update(kw)
    return B.PagedParams(**base)


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def decode(lib, p, Q=A, qs=0, Kc=A, Vc=A, table=A, n=A, O=A, ws=A, nbytes=1 << 40):
    return lib.blossom_attn_decode(ctypes.byref(p.c()) if p else None, Q, qs, Kc, Vc, table, n, O, None, ws, nbytes, None)


def prompt(lib, p, Q=A, qs=0, Kc=A, Vc=A, table=A, cu=A, n=A, O=A, ws=A, nbytes=1 << 40):
    return lib.blossom_attn_prompt(ctypes.byref(p.c()) if p else None, Q, qs, Kc, Vc, table, cu, n, O, None, ws, nbytes, None)


def append(lib, p, Q=A, qs=0, K=A, ks=0, V=A, vs=0, cos=A, sin=A, table=A, cu=A, n=A, Kc=A, Vc=A, Qr=A):
    return lib.blossom_kv_append(ctypes.byref(p.c()) if p else None, Q, qs, K, ks, V, vs, cos, sin, table, cu, n, Kc, Vc, Qr, None)


BAD = [(dict(S=0), -2), (dict(T=0), -2), (dict(H=0), -2), (dict(G=0), -2), (dict(n_pages=0), -2), (dict(max_pages=0), -2),
       (dict(max_pages=1 << 27), -2), (dict(T=1 << 29, H=4), -2), (dict(S=1 << 29, H=4), -2),
       (dict(d=48), -3), (dict(d=256), -3), (dict(page=4), -3), (dict(page=24), -3), (dict(page=512), -3), (dict(dtype=2), -3),
       (dict(G=3), -4), (dict(window=-1), -4), (dict(max_len=-1), -4), (dict(table_per_head=2), -4),
       (dict(softmax_scale=-1.0), -4), (dict(softmax_scale=float("nan")), -4), (dict(softmax_scale=float("inf")), -4)]


@pytest.mark.parametrize("change,code", BAD)
def test_bad_parameters(lib, change, code):
    p = params(**change)
    assert decode(lib, p) == code and prompt(lib, p) == code and append(lib, p) == code
    assert B.paged_workspace_bytes(p, B.WS_DECODE) == 0 and B.paged_workspace_bytes(p, B.WS_PROMPT) == 0


def test_missing_and_misaligned_pointers(lib):
    p, off = params(), vp(4104)
    assert decode(lib, None) == -1 and prompt(lib, None) == -1 and append(lib, None) == -1
    for name in ("Q", "Kc", "Vc", "table", "n", "O"):
        assert decode(lib, p, **{name: None}) == -1 and prompt(lib, p, **{name: None}) == -1, name
    assert prompt(lib, p, cu=None) == -1
    for name in ("Q", "Kc", "Vc", "O"):
        assert decode(lib, p, **{name: off}) == -5 and prompt(lib, p, **{name: off}) == -5, name
    for name in ("K", "V", "table", "cu", "n", "Kc", "Vc"):
        assert append(lib, p, **{name: None}) == -1, name
    # queries go with their output and with the tables, the tables with each other
    for name in ("Q", "Qr", "cos", "sin"):
        assert append(lib, p, **{name: None}) == -1, name
    assert append(lib, p, cos=None, sin=None) == -1
    for name in ("Q", "K", "V", "cos", "sin", "Kc", "Vc", "Qr"):
        assert append(lib, p, **{name: off}) == -5, name


def test_strides(lib):
    p = params()
    for call, name, row in ((decode, "qs", 256), (prompt, "qs", 256), (append, "qs", 256), (append, "ks", 128), (append, "vs", 128)):
        assert call(lib, p, **{name: row - 8}) == -4 and call(lib, p, **{name: -row}) == -4, (call, name)
        assert call(lib, p, **{name: row + 4}) == -5, (call, name)
    assert decode(lib, params(dtype=B.F32), qs=256 + 2) == -5


def test_per_head_tables_are_decodes(lib):
    p = params(table_per_head=1)
    assert prompt(lib, p) == -3 and append(lib, p) == -3 and decode(lib, p, Q=None) == -1


def test_workspace(lib):
    p = params(S=1, max_pages=4096)
    need = B.paged_workspace_bytes(p, B.WS_DECODE)
    # parts of four heads' rows: sums, reference, sum of exponentials; and where the sequence's parts begin, and how many
    assert need > 0 and (need - 8) % (4 * 4 * (64 + 2)) == 0
    assert decode(lib, p, ws=None) == -6 and decode(lib, p, nbytes=need - 1) == -6 and decode(lib, p, ws=vp(4104)) == -5
    assert B.paged_workspace_bytes(p, B.WS_FWD) == 0 and B.paged_workspace_bytes(p, 99) == 0
    assert B.workspace_bytes(B.Params(1, 1, 8, 8, 8, 1, 1), B.WS_DECODE) == 0
    # a window, a capacity: no parts for keys that nobody sees
    assert B.paged_workspace_bytes(params(S=1, max_pages=4096, window=16), B.WS_DECODE) == 0
    assert B.paged_workspace_bytes(params(S=1, max_pages=4096, max_len=16), B.WS_DECODE) == 0


def test_capacity():
    assert params().capacity == 64 and params(max_len=50).capacity == 50 and params(max_len=100).capacity == 64


def test_the_binding_names_what_is_wrong():
    p = params()
    z = torch.zeros
    bf = torch.bfloat16
    ok = dict(K_cache=z(10, 2, 16, 64, dtype=bf), V_cache=z(10, 2, 16, 64, dtype=bf), page_table=z(2, 4, dtype=torch.int32),
              kv_len=z(2, dtype=torch.int32))
    cu = z(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="^Q: expected cuda tensor"):
        B.attn_decode(p, z(2, 4, 64, dtype=bf), O=z(2, 4, 64, dtype=bf), **ok)
    with pytest.raises(ValueError, match="^Q is required"):
        B.attn_decode(p, None, **ok)
    with pytest.raises(ValueError, match="cu_seqlens is required"):
        B.attn_prompt(p, z(6, 4, 64, dtype=bf), cu_seqlens=None, **ok)
    with pytest.raises(ValueError, match="^K: expected cuda tensor"):
        B.kv_append(p, z(6, 2, 64, dtype=bf), z(6, 2, 64, dtype=bf), cu_seqlens=cu, **ok)


@pytest.mark.parametrize("dtype,size", [(B.F32, 4), (B.BF16, 2)])
@pytest.mark.parametrize("d", [8, 16, 32, 64, 128])
def test_decode_parts_stay_within_a_round_of_workgroups(dtype, size, d):
    # the join holds a weight for each of 256 parts; what is lost to rounding up is a part a sequence, so there are two for each at least
    seen = set()
    for S in (1, 2, 3, 7, 16, 64, 65, 100, 127, 128, 129, 200, 1000, 5000):
        for H, G in ((1, 1), (2, 1), (2, 2), (8, 2), (17, 1), (32, 8), (40, 1), (64, 64)):
            for positions in (32, 128, 512, 1024, 4096, 65536, 1 << 20, 1 << 24):
                p = params(S=S, H=H, G=G, d=d, dtype=dtype, page=16, n_pages=1, max_pages=positions // 16)
                need = B.paged_workspace_bytes(p, B.WS_DECODE)
                if need:
                    parts, rest = divmod(need - 8 * S, H * (d + 2) * 4)
                    assert rest == 0 and 2 * S <= parts <= 256, p
                    seen.add(parts)
    assert 256 in seen and min(seen) < 64


def test_calls_of_more_threads_than_a_launch_counts(lib):
    # a wavefront a token (append), four a sequence and key/value head (decode), two for 32 rows (prompts of small rows), four for 64
    for T, d in ((1 << 26, 64), (1 << 30, 64), (1 << 26, 8)):
        assert append(lib, params(T=T, H=1, G=1, d=d)) == -2, T
    for S, d in ((1 << 24, 64), (1 << 30, 64), (1 << 24, 8)):
        assert decode(lib, params(S=S, H=1, G=1, d=d, max_pages=2)) == -2, S
    for T, H, dtype, d in ((1 << 30, 1, B.F32, 8), (1 << 29, 2, B.F32, 64), (1 << 28, 4, B.BF16, 16)):
        assert prompt(lib, params(T=T, H=H, G=1, d=d, dtype=dtype)) == -2, T
    assert prompt(lib, params(S=1 << 25, T=1 << 10, H=1, G=1, d=64)) == -2
