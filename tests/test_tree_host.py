"""Refusals of trees, forks and beams before anything touches a GPU: the C entry points' codes, and the binding's messages on both of its paths."""
import ctypes
import types

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2512_13368_amd import binding as B
from test_paged_host import BAD, params

vp = ctypes.c_void_p
A, A2, A3 = vp(4096), vp(8192), vp(12288)  # fake addresses: every call must fail before they are used
STREAM = types.SimpleNamespace(cuda_stream=0)

pytestmark = pytest.mark.filterwarnings("ignore::UserWarning")


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def at(p):
    return ctypes.byref(p.c()) if p else None


def tree(lib, p, Q=A, qs=0, Kc=A, Vc=A, table=A, cu=A, n=A, mask=A, O=A, ws=A, nbytes=1 << 40):
    return lib.blossom_attn_tree(at(p), Q, qs, Kc, Vc, table, cu, n, mask, O, None, ws, nbytes, None)


def append(lib, p, Q=A, qs=0, K=A, ks=0, V=A, vs=0, cos=A, sin=A, table=A, cu=A, n=A, mask=A, Kc=A, Vc=A, Qr=A):
    return lib.blossom_kv_append_tree(at(p), Q, qs, K, ks, V, vs, cos, sin, table, cu, n, mask, Kc, Vc, Qr, None)


def accept(lib, p, width=4, keep=A, table=A, cu=A, n=A, Kc=A, Vc=A, out=A2):
    return lib.blossom_kv_accept(at(p), width, keep, table, cu, n, Kc, Vc, out, None)


def fork(lib, p, N=3, grow=1, parent=A, table=A, n=A, refs=A, to=A2, out=A2, new_refs=A2, copies=A3, missing=A3, ws=A, nbytes=1 << 40):
    return lib.blossom_kv_fork(at(p), N, grow, parent, table, n, refs, to, out, new_refs, copies, missing, ws, nbytes, None)


def copy(lib, p, count=3, copies=A, Kc=A, Vc=A):
    return lib.blossom_kv_copy_pages(at(p), count, copies, Kc, Vc, None)


def beam(lib, p, logits=A, stride=0, score=A, ended=None, parent=A, token=A, out=A, ends=None, ws=A, nbytes=1 << 40):
    return lib.blossom_beam_select(at(p), logits, stride, score, ended, parent, token, out, ends, ws, nbytes, None)


CALLS = [tree, append, accept, fork, copy]


@pytest.mark.parametrize("change,code", BAD)
def test_bad_parameters(lib, change, code):
    p = params(**change)
    for call in CALLS:
        assert call(lib, p) == code, call
    assert B.paged_workspace_bytes(p, B.WS_TREE) == 0 and B.fork_workspace_bytes(p, 3) == 0


def test_tables_per_head_are_refused(lib):
    p = params(table_per_head=1)
    assert [call(lib, p) for call in (tree, append, accept, fork)] == [-3] * 4


def test_missing_pointers(lib):
    p = params()
    for call in CALLS:
        assert call(lib, None) == -1
    needed = {tree: ("Q", "Kc", "Vc", "table", "cu", "n", "mask", "O"), append: ("K", "V", "table", "cu", "n", "mask", "Kc", "Vc", "cos", "sin", "Qr", "Q"),
              accept: ("keep", "table", "cu", "n", "Kc", "Vc"), copy: ("copies", "Kc", "Vc"),
              fork: ("parent", "table", "n", "refs", "to", "out", "new_refs", "copies", "missing")}
    for call, names in needed.items():
        for name in names:
            assert call(lib, p, **{name: None}) == -1, (call, name)


def test_misaligned_pointers_and_strides(lib):
    p, off = params(), vp(4104)
    for name in ("Q", "Kc", "Vc", "O"):
        assert tree(lib, p, **{name: off}) == -5, name
    for name in ("Q", "K", "V", "Kc", "Vc", "cos", "sin", "Qr"):
        assert append(lib, p, **{name: off}) == -5, name
    for call in (tree, append):
        assert call(lib, p, mask=vp(4100)) == -5
        assert call(lib, p, qs=100) == -4 and call(lib, p, qs=257) == -5
    for name in ("Kc", "Vc"):
        assert accept(lib, p, **{name: off}) == -5 and copy(lib, p, **{name: off}) == -5
    assert fork(lib, p, ws=off) == -5


def test_sizes_and_workspaces(lib):
    p = params()
    assert accept(lib, p, width=0) == -2 and copy(lib, p, count=0) == -2 and fork(lib, p, N=0) == -2
    assert fork(lib, p, grow=-1) == -4
    assert fork(lib, params(max_pages=1 << 20), N=1 << 12) == -2
    need = B.fork_workspace_bytes(p, 3)
    assert need > 0 and fork(lib, p, nbytes=need - 1) == -6 and fork(lib, p, ws=None) == -6 and B.fork_workspace_bytes(p, 0) == 0
    wide = params(S=1, T=20, max_pages=4096)
    need = B.paged_workspace_bytes(wide, B.WS_TREE)
    assert need > 0 and tree(lib, wide, nbytes=need - 1) == -6 and tree(lib, wide, ws=None) == -6 and tree(lib, wide, ws=vp(4104)) == -5
    assert B.paged_workspace_bytes(p, 7) == 0


def test_outputs_that_are_inputs_are_refused(lib):
    p = params()
    assert accept(lib, p, n=A, out=A) == -4
    assert fork(lib, p, table=A, to=A) == -4 and fork(lib, p, n=A, out=A) == -4 and fork(lib, p, refs=A, new_refs=A) == -4


def test_calls_of_more_threads_than_a_launch_counts(lib):
    assert tree(lib, params(T=1 << 24, H=64, G=64, max_pages=1, dtype=0)) == -2
    assert append(lib, params(T=1 << 28, max_pages=1)) == -2
    assert accept(lib, params(S=1 << 24)) == -2
    assert copy(lib, params(), count=1 << 24) == -2
    assert fork(lib, params(max_pages=1), N=1 << 26) == -2
    assert fork(lib, params(n_pages=(1 << 30) + 1)) == -2


BEAM_BAD = [(dict(B=0), -2), (dict(W=0), -2), (dict(K=0), -2), (dict(V=0), -2), (dict(W=65), -3), (dict(K=65), -3), (dict(dtype=2), -3),
            (dict(B=1 << 26), -2), (dict(eos=-2), -4), (dict(eos=100), -4)]


def test_beam_refusals(lib):
    def bp(**kw):
        return B.BeamParams(**{**dict(B=2, W=3, K=4, V=100), **kw})

    for change, code in BEAM_BAD:
        assert beam(lib, bp(**change)) == code, change
        assert B.beam_workspace_bytes(bp(**change)) == 0
    p = bp()
    assert beam(lib, None) == -1
    for name in ("logits", "score", "parent", "token", "out"):
        assert beam(lib, p, **{name: None}) == -1, name
        assert beam(lib, p, **{name: vp(4097)}) == -5, name
    assert beam(lib, p, stride=99) == -4 and beam(lib, p, stride=-1) == -4
    assert beam(lib, p, ended=A) == -4  # without an item that ends
    need = B.beam_workspace_bytes(p)
    assert need > 0 and beam(lib, p, nbytes=need - 1) == -6 and beam(lib, p, ws=None) == -6 and beam(lib, p, ws=vp(4104)) == -5
    assert beam(lib, bp(B=1 << 24, W=1, K=1)) == -2


# ---- the binding: stand-ins without memory take the tensors' places ----

P = params()


def dev(*shape, dtype=torch.bfloat16):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device="cuda")


def i32(*shape):
    return dev(*shape, dtype=torch.int32)


def tensors():
    p, f32 = P, torch.float32
    cache = (p.n_pages, p.G, p.page, p.d)
    rope = (p.capacity, p.d // 2)
    return {
        "attn_tree": dict(Q=dev(p.T, p.H, p.d), K_cache=dev(*cache), V_cache=dev(*cache), page_table=i32(p.S, p.max_pages), cu_seqlens=i32(p.S + 1),
                          kv_len=i32(p.S), tree_mask=dev(p.T, dtype=torch.int64), O=dev(p.T, p.H, p.d)),
        "kv_append_tree": dict(K=dev(p.T, p.G, p.d), V=dev(p.T, p.G, p.d), K_cache=dev(*cache), V_cache=dev(*cache), page_table=i32(p.S, p.max_pages),
                               cu_seqlens=i32(p.S + 1), kv_len=i32(p.S), tree_mask=dev(p.T, dtype=torch.int64), Q=dev(p.T, p.H, p.d),
                               rope=(dev(*rope, dtype=f32), dev(*rope, dtype=f32)), Q_rot=dev(p.T, p.H, p.d)),
        "kv_accept": dict(keep=i32(p.S, 5), K_cache=dev(*cache), V_cache=dev(*cache), page_table=i32(p.S, p.max_pages), cu_seqlens=i32(p.S + 1),
                          kv_len=i32(p.S), new_len=i32(p.S)),
        "kv_fork": dict(parent=i32(7), page_table=i32(p.S, p.max_pages), kv_len=i32(p.S), refs=i32(p.n_pages), grow=1, new_table=i32(7, p.max_pages),
                        new_len=i32(7), new_refs=i32(p.n_pages), copies=i32(7, 3), missing=i32(1), ws=dev(1 << 12, dtype=torch.uint8)),
        "kv_copy_pages": dict(copies=i32(7, 3), K_cache=dev(*cache), V_cache=dev(*cache)),
        "beam_select": dict(logits=dev(6, 100), score=dev(2, 3, dtype=f32), ended=dev(2, 3, dtype=torch.bool), parent=i32(2, 4), token=i32(2, 4),
                            out_score=dev(2, 4, dtype=f32), out_ended=dev(2, 4, dtype=torch.bool), ws=dev(1 << 16, dtype=torch.uint8)),
    }


def call(name, a):
    p = B.BeamParams(B=2, W=3, K=4, V=100, dtype=B.BF16, eos=1) if name == "beam_select" else P
    return getattr(B, name)(p, **a, stream=STREAM)


@pytest.fixture(params=["compiled", "python"])
def path(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(B, "_fast", B.PYTHON_PATH)
    else:
        assert B.fastcall() is not B.PYTHON_PATH
    return request.param


NAMES = list(tensors())


@pytest.mark.parametrize("name", NAMES)
def test_the_stand_ins_reach_the_library(path, name):
    with pytest.raises(B.BlossomError) as e:
        call(name, tensors()[name])
    assert e.value.code == -1


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_shape_type_or_layout_are_refused(path, name):
    for key, t in tensors()[name].items():
        if not isinstance(t, torch.Tensor):
            continue
        wrong = [dev(*t.shape, 2, dtype=t.dtype), dev(*t.shape, dtype=torch.float64)]
        if key != "ws":
            wrong.append(torch.empty(t.shape, dtype=t.dtype))  # host memory
        if t.dim() == 2 and key not in ("logits",):
            wrong.append(dev(t.shape[1], t.shape[0], dtype=t.dtype).t())
        for w in wrong if key != "ws" else [torch.empty(1 << 16, dtype=torch.uint8)]:
            with pytest.raises(ValueError):
                call(name, {**tensors()[name], key: w})


@pytest.mark.parametrize("name", NAMES)
def test_missing_tensors_are_named(path, name):
    optional = {"O", "Q", "Q_rot", "rope", "new_len", "new_table", "new_refs", "copies", "missing", "ws", "ended", "parent", "token", "out_score", "out_ended", "grow"}
    if name == "kv_fork":
        optional -= {"parent"}
    if name == "kv_copy_pages":
        optional -= {"copies"}
    if name == "attn_tree":
        optional -= {"Q"}
    for key in set(tensors()[name]) - optional:
        with pytest.raises(ValueError, match=key):
            call(name, {**tensors()[name], key: None})


def test_rows_of_logits_that_overlap_are_refused(path):
    a = tensors()["beam_select"]
    for bad in (a["logits"][:1].expand(6, 100), a["logits"].as_strided((6, 100), (50, 1)), a["logits"].as_strided((6, 100), (1, 6))):
        with pytest.raises(ValueError, match="^logits"):
            call("beam_select", {**a, "logits": bad})
    wide = dev(6, 128)[:, :100]
    with pytest.raises(B.BlossomError) as e:
        call("beam_select", {**a, "logits": wide})
    assert e.value.code == -1


def test_counts_beyond_32_bits_are_refused(path):
    # (they would wrap round to small ones)
    a = tensors()
    for name, key, wrong in (("kv_accept", "keep", i32(P.S, (1 << 32) + 5)), ("kv_copy_pages", "copies", i32((1 << 32) + 7, 3)),
                             ("kv_fork", "grow", (1 << 32) + 1), ("kv_fork", "grow", -(1 << 32) + 1)):
        with pytest.raises(ValueError, match=key):
            call(name, {**a[name], key: wrong})
    with pytest.raises(ValueError, match="parent"):
        B.kv_fork(P, i32((1 << 32) + 7), a["kv_fork"]["page_table"], a["kv_fork"]["kv_len"], a["kv_fork"]["refs"])
