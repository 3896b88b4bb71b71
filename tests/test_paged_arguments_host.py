"""What the paged cache's calls refuse in tensors that look like device tensors of the right shape and type, on both paths of the binding.
Stand-ins without memory take the tensors' places: a call that gets as far as the library ends with its error of a missing pointer."""
import types

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2512_13368_amd import binding as B

STREAM = types.SimpleNamespace(cuda_stream=0)
BF = torch.bfloat16
P = B.PagedParams(S=2, T=6, H=4, G=2, d=64, page=16, n_pages=10, max_pages=4, dtype=B.BF16)

pytestmark = pytest.mark.filterwarnings("ignore::UserWarning")


def dev(*shape, dtype=BF):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device="cuda")


def arguments(p=P):
    """Every tensor that the three calls take, in order."""
    i32 = torch.int32
    return dict(Q=dev(p.T, p.H, p.d), K=dev(p.T, p.G, p.d), V=dev(p.T, p.G, p.d), K_cache=dev(p.n_pages, p.G, p.page, p.d),
                V_cache=dev(p.n_pages, p.G, p.page, p.d), page_table=dev(p.S, p.max_pages, dtype=i32), cu_seqlens=dev(p.S + 1, dtype=i32),
                kv_len=dev(p.S, dtype=i32), O=dev(p.T, p.H, p.d), one=dev(p.S, p.H, p.d), one_O=dev(p.S, p.H, p.d),
                rope=(dev(p.capacity, p.d // 2, dtype=torch.float32), dev(p.capacity, p.d // 2, dtype=torch.float32)))


def append(a, p=P):
    return B.kv_append(p, a["K"], a["V"], a["K_cache"], a["V_cache"], a["page_table"], a["cu_seqlens"], a["kv_len"], Q=a["Q"],
                       rope=a["rope"], Q_rot=a["O"], stream=STREAM)


def decode(a, p=P, ws=None):
    return B.attn_decode(p, a["one"], a["K_cache"], a["V_cache"], a["page_table"], a["kv_len"], O=a["one_O"], ws=ws, stream=STREAM)


def prompt(a, p=P, ws=None):
    return B.attn_prompt(p, a["Q"], a["K_cache"], a["V_cache"], a["page_table"], a["cu_seqlens"], a["kv_len"], O=a["O"], ws=ws, stream=STREAM)


@pytest.fixture(params=["compiled", "python"])
def path(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(B, "_fast", B.PYTHON_PATH)
    else:
        assert B.fastcall() is not B.PYTHON_PATH
    return request.param


@pytest.mark.parametrize("call", [append, decode, prompt])
def test_the_stand_ins_reach_the_library(call):
    with pytest.raises(B.BlossomError) as e:
        call(arguments())
    assert e.value.code == -1


@pytest.mark.parametrize("call,name", [(append, "Q"), (append, "K"), (append, "V"), (decode, "one"), (prompt, "Q")])
@pytest.mark.parametrize("kind", ["expanded", "overlapping"])
def test_tokens_that_share_memory_are_refused(path, call, name, kind):
    # a token stride of 0 would be taken for rows one after another, in memory that holds a single one
    a = arguments()
    t = a[name]
    a[name] = t[:1].expand(*t.shape) if kind == "expanded" else t.as_strided(t.shape, (t.shape[2] * (t.shape[1] - 1), t.shape[2], 1))
    with pytest.raises(ValueError, match="^[QKV]: .* tokens that do not overlap"):
        call(a)


@pytest.mark.parametrize("call,name", [(append, "Q"), (append, "K"), (append, "V"), (decode, "one"), (prompt, "Q")])
def test_a_single_token_may_have_any_stride(call, name):
    p = B.PagedParams(**{**P.__dict__, "S": 1, "T": 1})
    a = arguments(p)
    a[name] = a[name].as_strided(a[name].shape, (0, p.d, 1))
    with pytest.raises(B.BlossomError) as e:
        call(a, p)
    assert e.value.code == -1


LONG = B.PagedParams(**{**P.__dict__, "S": 1, "T": 1, "n_pages": 5000, "max_pages": 4096})  # a split, and so a workspace


def no_workspaces(need):
    """Tensors of `need` bytes or more that are not memory of the GPU, or not as much of it as they have elements."""
    with FakeTensorMode():
        small = torch.empty(1, dtype=torch.uint8, device="cuda")
        wide = torch.empty(2 * need, dtype=torch.uint8, device="cuda")
    return {"host memory": torch.empty(need + 64, dtype=torch.uint8), "expanded": small.expand(need + 64), "every other byte": wide[::2]}


@pytest.mark.parametrize("kind", ["host memory", "expanded", "every other byte"])
@pytest.mark.parametrize("call,which", [(decode, B.WS_DECODE), (prompt, B.WS_PROMPT)])
def test_workspaces_that_are_no_device_memory_are_refused(path, call, which, kind):
    need = B.paged_workspace_bytes(LONG, which)
    assert need > 0
    with pytest.raises(ValueError, match="^ws: expected contiguous cuda tensor"):
        call(arguments(LONG), LONG, ws=no_workspaces(need)[kind])


@pytest.mark.parametrize("call", [decode, prompt])
def test_a_workspace_that_nobody_needs_may_be_anything(call):
    assert B.paged_workspace_bytes(P, B.WS_DECODE) == 0 and B.paged_workspace_bytes(P, B.WS_PROMPT) == 0
    with pytest.raises(B.BlossomError) as e:
        call(arguments(), ws=torch.empty(16, dtype=torch.uint8))
    assert e.value.code == -1


@pytest.mark.parametrize("kind", ["host memory", "expanded", "every other byte"])
def test_selection_refuses_such_workspaces_too(path, kind):
    p = B.Params(2, 2, 128, 32, 8, 4, 16, B.F32)
    f = torch.float32
    Q, K, valid, sel = dev(2, 2, 128, 32, dtype=f), dev(2, 2, 128, 32, dtype=f), dev(2, dtype=torch.int32), dev(2, 2, p.NB, 4, dtype=torch.int32)
    need = B.workspace_bytes(p, B.WS_SELECT)
    assert need > 0
    with pytest.raises(ValueError, match="^ws: expected contiguous cuda tensor"):
        B.select_blocks(p, Q, K, valid, sel=sel, ws=no_workspaces(need)[kind], stream=STREAM)
