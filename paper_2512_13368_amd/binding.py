"""Python binding of libblossom.so: argument marshalling only (that of the hot calls in native code, ``_fastcall.so``).

Every step of the path runs in the HIP kernels behind the C ABI of
``include/blossom.h``; this module turns torch device tensors into pointers,
allocates outputs and workspaces with torch, and raises on error codes.  There
is no CPU fallback: a missing library is an ImportError-like failure.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libblossom.so")

F32, BF16 = 0, 1
WS_SELECT, WS_FWD, WS_BWD, WS_DENSE, WS_DECODE, WS_PROMPT, WS_TREE = 0, 1, 2, 3, 4, 5, 6

EXPORTS = ("blossom_workspace_bytes", "blossom_select_blocks", "blossom_select_blocks_static", "blossom_select_blocks_cmp",
           "blossom_rope_select_blocks", "blossom_attn_bwd_rope", "blossom_select_positions_workspace_bytes",
           "blossom_select_positions", "blossom_attn_fwd_positions", "blossom_attn_bwd_positions", "blossom_out_proj_ln", "blossom_attn_fwd", "blossom_attn_bwd",
           "blossom_attn_bwd_stages", "blossom_paged_workspace_bytes", "blossom_kv_append", "blossom_attn_decode", "blossom_attn_prompt",
           "blossom_kv_append_tree", "blossom_attn_tree", "blossom_kv_accept", "blossom_fork_workspace_bytes", "blossom_kv_fork",
           "blossom_kv_copy_pages", "blossom_beam_workspace_bytes", "blossom_beam_select",
           "blossom_dense_causal_fwd", "blossom_probe_bytes", "blossom_probe", "blossom_strerror", "blossom_version")
PROBE_WORKGROUPS = 4096
BWD_GATE, BWD_INVERSE, BWD_DQ, BWD_DKV, BWD_ALL = 1, 2, 4, 8, 15


class BlossomParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("d", ctypes.c_int32),
                ("block", ctypes.c_int32), ("topk", ctypes.c_int32), ("window", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("stis_mode", ctypes.c_int32), ("save_for_bwd", ctypes.c_int32),
                ("stis_block", ctypes.c_int32), ("last_block_only", ctypes.c_int32)]


class BlossomPagedParams(ctypes.Structure):
    _fields_ = [(name, ctypes.c_float if name == "softmax_scale" else ctypes.c_int32)
                for name in ("S", "T", "H", "G", "d", "page", "n_pages", "max_pages", "dtype", "softmax_scale", "window", "max_len",
                             "table_per_head")]


class BlossomBeamParams(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("B", "W", "K", "V", "dtype", "eos")]


class BlossomError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


_lib = None


def lib() -> ctypes.CDLL:
    """Open libblossom.so (after torch, so that both use one HIP runtime instance)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`"
                " (there is no fallback path)")
        import torch  # noqa: F401  (loads torch's HIP runtime first)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p, fp = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
        pp = ctypes.POINTER(BlossomParams)
        L.blossom_workspace_bytes.restype = ctypes.c_size_t
        L.blossom_workspace_bytes.argtypes = [pp, ctypes.c_int]
        L.blossom_select_blocks.restype = ctypes.c_int
        L.blossom_select_blocks.argtypes = [pp, vp, vp, i32p, i32p, vp, ctypes.c_size_t, vp]
        L.blossom_select_blocks_static.restype = ctypes.c_int
        L.blossom_select_blocks_static.argtypes = [pp, vp, vp, i32p, i32p, vp]
        L.blossom_rope_select_blocks.restype = ctypes.c_int
        L.blossom_rope_select_blocks.argtypes = [pp, vp, vp, fp, fp, i32p, vp, vp, i32p, vp, ctypes.c_size_t, vp]
        L.blossom_select_positions_workspace_bytes.restype = ctypes.c_size_t
        L.blossom_select_positions_workspace_bytes.argtypes = [pp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        L.blossom_select_positions.restype = ctypes.c_int
        L.blossom_select_positions.argtypes = [pp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                               vp, vp, i32p, i32p, vp, ctypes.c_size_t, vp]
        L.blossom_attn_fwd_positions.restype = ctypes.c_int
        L.blossom_attn_fwd_positions.argtypes = [pp, ctypes.c_int32] + [vp] * 12 + [vp]
        L.blossom_attn_bwd_positions.restype = ctypes.c_int
        L.blossom_attn_bwd_positions.argtypes = [pp, ctypes.c_int32, vp, vp, vp, i32p, i32p, fp, fp, vp, vp, fp, fp, vp, vp,
                                                 vp, vp, fp, fp, vp, ctypes.c_size_t, vp]
        L.blossom_out_proj_ln.restype = ctypes.c_int
        L.blossom_out_proj_ln.argtypes = [pp, ctypes.c_int32, vp, vp, fp, vp, fp, fp, ctypes.c_float, vp, fp, fp, vp]
        L.blossom_select_blocks_cmp.restype = ctypes.c_int
        L.blossom_select_blocks_cmp.argtypes = [pp, vp, vp, i32p, i32p, vp, ctypes.c_size_t, vp]
        L.blossom_attn_fwd.restype = ctypes.c_int
        L.blossom_attn_fwd.argtypes = [pp, vp, vp, vp, i32p, i32p, fp, fp, vp, vp, vp, fp, fp, vp,
                                       ctypes.c_size_t, vp]
        L.blossom_attn_bwd.restype = ctypes.c_int
        L.blossom_attn_bwd.argtypes = [pp, vp, vp, vp, i32p, i32p, fp, fp, vp, vp, fp, fp, vp, vp, vp, vp,
                                       fp, fp, vp, ctypes.c_size_t, vp]
        L.blossom_attn_bwd_rope.restype = ctypes.c_int
        L.blossom_attn_bwd_rope.argtypes = [pp, vp, vp, vp, i32p, i32p, fp, fp, vp, vp, fp, fp, vp, fp, fp, vp, vp, vp,
                                            fp, fp, vp, ctypes.c_size_t, vp]
        L.blossom_attn_bwd_stages.restype = ctypes.c_int
        L.blossom_attn_bwd_stages.argtypes = L.blossom_attn_bwd.argtypes + [ctypes.c_uint]
        gp, i64 = ctypes.POINTER(BlossomPagedParams), ctypes.c_int64
        L.blossom_paged_workspace_bytes.restype = ctypes.c_size_t
        L.blossom_paged_workspace_bytes.argtypes = [gp, ctypes.c_int]
        L.blossom_kv_append.restype = ctypes.c_int
        L.blossom_kv_append.argtypes = [gp, vp, i64, vp, i64, vp, i64, fp, fp, i32p, i32p, i32p, vp, vp, vp, vp]
        L.blossom_attn_decode.restype = ctypes.c_int
        L.blossom_attn_decode.argtypes = [gp, vp, i64, vp, vp, i32p, i32p, vp, fp, vp, ctypes.c_size_t, vp]
        L.blossom_attn_prompt.restype = ctypes.c_int
        L.blossom_attn_prompt.argtypes = [gp, vp, i64, vp, vp, i32p, i32p, i32p, vp, fp, vp, ctypes.c_size_t, vp]
        L.blossom_kv_append_tree.restype = ctypes.c_int
        L.blossom_kv_append_tree.argtypes = [gp, vp, i64, vp, i64, vp, i64, fp, fp, i32p, i32p, i32p, vp, vp, vp, vp, vp]
        L.blossom_attn_tree.restype = ctypes.c_int
        L.blossom_attn_tree.argtypes = [gp, vp, i64, vp, vp, i32p, i32p, i32p, vp, vp, fp, vp, ctypes.c_size_t, vp]
        L.blossom_kv_accept.restype = ctypes.c_int
        L.blossom_kv_accept.argtypes = [gp, ctypes.c_int32, i32p, i32p, i32p, i32p, vp, vp, i32p, vp]
        L.blossom_fork_workspace_bytes.restype = ctypes.c_size_t
        L.blossom_fork_workspace_bytes.argtypes = [gp, ctypes.c_int32]
        L.blossom_kv_fork.restype = ctypes.c_int
        L.blossom_kv_fork.argtypes = [gp, ctypes.c_int32, ctypes.c_int32] + [i32p] * 9 + [vp, ctypes.c_size_t, vp]
        L.blossom_kv_copy_pages.restype = ctypes.c_int
        L.blossom_kv_copy_pages.argtypes = [gp, ctypes.c_int32, i32p, vp, vp, vp]
        bp = ctypes.POINTER(BlossomBeamParams)
        L.blossom_beam_workspace_bytes.restype = ctypes.c_size_t
        L.blossom_beam_workspace_bytes.argtypes = [bp]
        L.blossom_beam_select.restype = ctypes.c_int
        L.blossom_beam_select.argtypes = [bp, vp, i64, fp, vp, i32p, i32p, fp, vp, vp, ctypes.c_size_t, vp]
        L.blossom_dense_causal_fwd.restype = ctypes.c_int
        L.blossom_dense_causal_fwd.argtypes = [pp, vp, vp, vp, i32p, vp, fp, vp, ctypes.c_size_t, vp]
        L.blossom_probe_bytes.restype = ctypes.c_size_t
        L.blossom_probe_bytes.argtypes = [ctypes.c_int]
        L.blossom_probe.restype = ctypes.c_int
        L.blossom_probe.argtypes = [ctypes.c_int, vp, vp, fp, ctypes.c_int, vp]
        L.blossom_strerror.restype = ctypes.c_char_p
        L.blossom_strerror.argtypes = [ctypes.c_int]
        L.blossom_version.restype = ctypes.c_char_p
        L.blossom_version.argtypes = []
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().blossom_strerror(int(code)).decode()


def version() -> str:
    return lib().blossom_version().decode()


@dataclass
class Params:
    B: int
    H: int
    L: int
    d: int
    block: int
    topk: int
    window: int
    dtype: int = F32
    softmax_scale: float = 0.0
    stis_mode: int = 0
    save_for_bwd: int = 0
    stis_block: int = 0
    last_block_only: int = 0

    @property
    def NB(self) -> int:
        return -(-self.L // self.block)

    def c(self) -> BlossomParams:
        return BlossomParams(self.B, self.H, self.L, self.d, self.block, self.topk, self.window,
                             self.dtype, self.softmax_scale, self.stis_mode, self.save_for_bwd, self.stis_block,
                             self.last_block_only)


class _PythonPath:
    """Stands in for the native marshalling: declines every call, so that the Python path below takes it."""

    def __getattr__(self, name):
        return lambda *args: None


PYTHON_PATH = _PythonPath()
_fast = None


def fastcall():
    """The native marshalling of the hot calls (csrc/fastcall.cpp).  Each returns the C ABI's error code, or None where an
    argument is missing or not as expected: then the Python path below allocates, or names what is wrong.  Without the
    module the Python path marshals every call, with the same kernels and results."""
    global _fast
    if _fast is None:
        import torch  # noqa: F401  (the module is linked against its libraries)
        lib()
        try:
            from . import _fastcall
            _fast = _fastcall
        except ImportError as e:
            import warnings
            warnings.warn(f"_fastcall.so cannot be loaded ({e}): calls are marshalled in Python, about 10 us each", RuntimeWarning)
            _fast = PYTHON_PATH
    return _fast


def workspace_bytes(p: Params, which: int) -> int:
    cp = p.c()
    return int(lib().blossom_workspace_bytes(ctypes.byref(cp), which))


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _torch_dtype(p: Params):
    import torch
    return torch.float32 if p.dtype == F32 else torch.bfloat16


def _check_tensor(t, shape, dtype, name):
    if t is None:
        return
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected contiguous cuda tensor {tuple(shape)} {dtype}, got "
                         f"{tuple(t.shape)} {t.dtype} contiguous={t.is_contiguous()} cuda={t.is_cuda}")


def _ws_bytes(ws, need: int) -> int:
    """Bytes of a caller's workspace, whose address goes to the device where `need` is not 0."""
    if ws is None:
        return 0
    if need and not (ws.is_cuda and ws.is_contiguous()):
        raise ValueError(f"ws: expected contiguous cuda tensor of {need} bytes or more, got {tuple(ws.shape)} {ws.dtype} "
                         f"contiguous={ws.is_contiguous()} cuda={ws.is_cuda}")
    return ws.numel() * ws.element_size()


def _workspace(p: Params, which: int, ws, device):
    import torch
    need = workspace_bytes(p, which)
    if ws is None and need > 0:
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    return ws, _ws_bytes(ws, need)


def select_blocks(p: Params, Q, K, valid_len, sel=None, ws=None, stream=None):
    rc = (_fast or fastcall()).select_blocks(p, Q, K, valid_len, sel, ws, stream)
    if rc is not None:
        if rc:
            raise BlossomError(rc, "blossom_select_blocks")
        return sel
    import torch
    shp = (p.B, p.H, p.L, p.d)
    _check_tensor(Q, shp, _torch_dtype(p), "Q")
    _check_tensor(K, shp, _torch_dtype(p), "K")
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    if sel is None:
        sel = torch.empty((p.B, p.H, p.NB, p.topk), dtype=torch.int32, device=Q.device)
    _check_tensor(sel, (p.B, p.H, p.NB, p.topk), torch.int32, "sel")
    ws, nbytes = _workspace(p, WS_SELECT, ws, Q.device)
    cp = p.c()
    rc = lib().blossom_select_blocks(ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(valid_len), _ptr(sel),
                                     _ptr(ws), nbytes, _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_select_blocks")
    return sel


def select_blocks_static(p: Params, Q, K, valid_len, sel, stream=None):
    """blossom_select_blocks_static: no workspace, nothing allocated (the caller passes `sel`)."""
    import torch
    shp = (p.B, p.H, p.L, p.d)
    _check_tensor(Q, shp, _torch_dtype(p), "Q")
    _check_tensor(K, shp, _torch_dtype(p), "K")
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    if sel is None:
        raise ValueError("sel is required: this entry point allocates nothing")
    _check_tensor(sel, (p.B, p.H, p.NB, p.topk), torch.int32, "sel")
    cp = p.c()
    rc = lib().blossom_select_blocks_static(ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(valid_len), _ptr(sel),
                                            _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_select_blocks_static")
    return sel


def rope_select_blocks(p: Params, Q, K, rope_cos, rope_sin, valid_len, Q_rot=None, K_rot=None, sel=None, ws=None,
                       stream=None):
    """blossom_rope_select_blocks: returns (Q_rot, K_rot, sel)."""
    rc = (_fast or fastcall()).rope_select_blocks(p, Q, K, rope_cos, rope_sin, valid_len, Q_rot, K_rot, sel, ws, stream)
    if rc is not None:
        if rc:
            raise BlossomError(rc, "blossom_rope_select_blocks")
        return Q_rot, K_rot, sel
    import torch
    shp = (p.B, p.H, p.L, p.d)
    dt = _torch_dtype(p)
    _check_tensor(Q, shp, dt, "Q")
    _check_tensor(K, shp, dt, "K")
    _check_tensor(rope_cos, (p.L, p.d // 2), torch.float32, "rope_cos")
    _check_tensor(rope_sin, (p.L, p.d // 2), torch.float32, "rope_sin")
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    if Q_rot is None:
        Q_rot = torch.empty(shp, dtype=dt, device=Q.device)
    if K_rot is None:
        K_rot = torch.empty(shp, dtype=dt, device=Q.device)
    _check_tensor(Q_rot, shp, dt, "Q_rot")
    _check_tensor(K_rot, shp, dt, "K_rot")
    if sel is None:
        sel = torch.empty((p.B, p.H, p.NB, p.topk), dtype=torch.int32, device=Q.device)
    _check_tensor(sel, (p.B, p.H, p.NB, p.topk), torch.int32, "sel")
    ws, nbytes = _workspace(p, WS_SELECT, ws, Q.device)
    cp = p.c()
    rc = lib().blossom_rope_select_blocks(ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(rope_cos), _ptr(rope_sin),
                                          _ptr(valid_len), _ptr(Q_rot), _ptr(K_rot), _ptr(sel), _ptr(ws), nbytes,
                                          _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_rope_select_blocks")
    return Q_rot, K_rot, sel


def select_blocks_cmp(p: Params, Q, Kcmp, valid_len, sel=None, ws=None, stream=None):
    """blossom_select_blocks_cmp: Kcmp [B,H,NB,d] holds the caller's compressed keys."""
    import torch
    _check_tensor(Q, (p.B, p.H, p.L, p.d), _torch_dtype(p), "Q")
    _check_tensor(Kcmp, (p.B, p.H, p.NB, p.d), _torch_dtype(p), "Kcmp")
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    if sel is None:
        sel = torch.empty((p.B, p.H, p.NB, p.topk), dtype=torch.int32, device=Q.device)
    _check_tensor(sel, (p.B, p.H, p.NB, p.topk), torch.int32, "sel")
    ws, nbytes = _workspace(p, WS_SELECT, ws, Q.device)
    cp = p.c()
    rc = lib().blossom_select_blocks_cmp(ctypes.byref(cp), _ptr(Q), _ptr(Kcmp), _ptr(valid_len), _ptr(sel),
                                         _ptr(ws), nbytes, _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_select_blocks_cmp")
    return sel


@dataclass
class FwdOut:
    O: object
    o_lt: object = None
    o_st: object = None
    lse_lt: object = None
    lse_st: object = None


def attn_fwd(p: Params, Q, K, V, valid_len, sel, gate_w, gate_b=None, out: FwdOut | None = None,
             ws=None, stream=None) -> FwdOut:
    if out is not None:
        rc = (_fast or fastcall()).attn_fwd(p, Q, K, V, valid_len, sel, gate_w, gate_b, out.O, out.o_lt, out.o_st, out.lse_lt,
                                            out.lse_st, ws, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_attn_fwd")
            return out
    import torch
    shp = (p.B, p.H, p.L, p.d)
    dt = _torch_dtype(p)
    for t, nm in ((Q, "Q"), (K, "K"), (V, "V")):
        _check_tensor(t, shp, dt, nm)
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    _check_tensor(sel, (p.B, p.H, p.NB, p.topk), torch.int32, "sel")
    _check_tensor(gate_w, (p.H, 2 * p.d), torch.float32, "gate_w")
    _check_tensor(gate_b, (p.H,), torch.float32, "gate_b")
    if out is None:
        out = FwdOut(torch.empty(shp, dtype=dt, device=Q.device))
        if p.save_for_bwd:
            out.o_lt = torch.empty(shp, dtype=torch.float32, device=Q.device)
            out.o_st = torch.empty(shp, dtype=torch.float32, device=Q.device)
            out.lse_lt = torch.empty(shp[:3], dtype=torch.float32, device=Q.device)
            out.lse_st = torch.empty(shp[:3], dtype=torch.float32, device=Q.device)
    _check_tensor(out.O, shp, dt, "O")
    _check_tensor(out.o_lt, shp, torch.float32, "o_lt")
    _check_tensor(out.o_st, shp, torch.float32, "o_st")
    _check_tensor(out.lse_lt, shp[:3], torch.float32, "lse_lt")
    _check_tensor(out.lse_st, shp[:3], torch.float32, "lse_st")
    ws, nbytes = _workspace(p, WS_FWD, ws, Q.device)
    cp = p.c()
    rc = lib().blossom_attn_fwd(ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(V), _ptr(valid_len), _ptr(sel),
                                _ptr(gate_w), _ptr(gate_b), _ptr(out.O), _ptr(out.o_lt), _ptr(out.o_st),
                                _ptr(out.lse_lt), _ptr(out.lse_st), _ptr(ws), nbytes, _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_attn_fwd")
    return out


@dataclass
class BwdOut:
    dQ: object
    dK: object
    dV: object
    d_gate_w: object
    d_gate_b: object


def attn_bwd(p: Params, Q, K, V, valid_len, sel, gate_w, gate_b, fwd: FwdOut, dO,
             out: BwdOut | None = None, ws=None, stream=None, stages: int = BWD_ALL, rope=None) -> BwdOut:
    """blossom_attn_bwd (or _stages); rope=(cos, sin) calls blossom_attn_bwd_rope instead."""
    if out is not None and stages == BWD_ALL:
        rc = (_fast or fastcall()).attn_bwd(p, Q, K, V, valid_len, sel, gate_w, gate_b, fwd.o_lt, fwd.o_st, fwd.lse_lt,
                                            fwd.lse_st, dO, out.dQ, out.dK, out.dV, out.d_gate_w, out.d_gate_b, ws,
                                            *(rope or (None, None)), stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_attn_bwd")
            return out
    import torch
    shp = (p.B, p.H, p.L, p.d)
    dt = _torch_dtype(p)
    for t, nm in ((Q, "Q"), (K, "K"), (V, "V"), (dO, "dO")):
        if t is None:
            raise ValueError(f"{nm} is required")
        _check_tensor(t, shp, dt, nm)
    for t, nm in ((fwd.o_lt, "o_lt"), (fwd.o_st, "o_st")):
        if t is None:
            raise ValueError(f"{nm} is required")
        _check_tensor(t, shp, torch.float32, nm)
    for t, nm in ((fwd.lse_lt, "lse_lt"), (fwd.lse_st, "lse_st")):
        if t is None:
            raise ValueError(f"{nm} is required")
        _check_tensor(t, shp[:3], torch.float32, nm)
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    _check_tensor(sel, (p.B, p.H, p.NB, p.topk), torch.int32, "sel")
    _check_tensor(gate_w, (p.H, 2 * p.d), torch.float32, "gate_w")
    _check_tensor(gate_b, (p.H,), torch.float32, "gate_b")
    if out is None:
        out = BwdOut(torch.empty(shp, dtype=dt, device=Q.device), torch.empty(shp, dtype=dt, device=Q.device),
                     torch.empty(shp, dtype=dt, device=Q.device),
                     torch.empty((p.H, 2 * p.d), dtype=torch.float32, device=Q.device),
                     torch.empty((p.H,), dtype=torch.float32, device=Q.device))
    for t, nm in ((out.dQ, "dQ"), (out.dK, "dK"), (out.dV, "dV")):
        _check_tensor(t, shp, dt, nm)
    _check_tensor(out.d_gate_w, (p.H, 2 * p.d), torch.float32, "d_gate_w")
    _check_tensor(out.d_gate_b, (p.H,), torch.float32, "d_gate_b")
    ws, nbytes = _workspace(p, WS_BWD, ws, Q.device)
    cp = p.c()
    args = (ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(V), _ptr(valid_len), _ptr(sel), _ptr(gate_w), _ptr(gate_b),
            _ptr(fwd.o_lt), _ptr(fwd.o_st), _ptr(fwd.lse_lt), _ptr(fwd.lse_st), _ptr(dO), _ptr(out.dQ),
            _ptr(out.dK), _ptr(out.dV), _ptr(out.d_gate_w), _ptr(out.d_gate_b), _ptr(ws), nbytes, _stream(stream))
    if rope is not None:
        _check_tensor(rope[0], (p.L, p.d // 2), torch.float32, "rope_cos")
        _check_tensor(rope[1], (p.L, p.d // 2), torch.float32, "rope_sin")
        if stages != BWD_ALL:
            raise ValueError("blossom_attn_bwd_rope runs all passes")
        rc = lib().blossom_attn_bwd_rope(*args[:13], _ptr(rope[0]), _ptr(rope[1]), *args[13:])
    elif stages == BWD_ALL:
        rc = lib().blossom_attn_bwd(*args)
    else:
        rc = lib().blossom_attn_bwd_stages(*args, stages)
    if rc:
        raise BlossomError(rc, "blossom_attn_bwd")
    return out


def dense_causal_fwd(p: Params, Q, K, V, valid_len, O=None, lse=None, ws=None, stream=None):
    import torch
    shp = (p.B, p.H, p.L, p.d)
    dt = _torch_dtype(p)
    for t, nm in ((Q, "Q"), (K, "K"), (V, "V")):
        _check_tensor(t, shp, dt, nm)
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    if O is None:
        O = torch.empty(shp, dtype=dt, device=Q.device)
    _check_tensor(O, shp, dt, "O")
    _check_tensor(lse, shp[:3], torch.float32, "lse")
    ws, nbytes = _workspace(p, WS_DENSE, ws, Q.device)
    cp = p.c()
    rc = lib().blossom_dense_causal_fwd(ctypes.byref(cp), _ptr(Q), _ptr(K), _ptr(V), _ptr(valid_len),
                                        _ptr(O), _ptr(lse), _ptr(ws), nbytes, _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_dense_causal_fwd")
    return O, lse


def probe_bytes(which: int) -> int:
    return int(lib().blossom_probe_bytes(which))


def probe(kind: int, K, V, sink, iters: int, stream=None):
    """blossom_probe: one launch of the stripped tile loop (the caller times it)."""
    rc = lib().blossom_probe(int(kind), _ptr(K), _ptr(V), _ptr(sink), int(iters), _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_probe")


def select_positions_workspace_bytes(p: Params, kv_groups: int, cmp_block: int, cmp_stride: int) -> int:
    cp = p.c()
    return int(lib().blossom_select_positions_workspace_bytes(ctypes.byref(cp), kv_groups, cmp_block, cmp_stride))


def select_positions(p: Params, kv_groups: int, cmp_block: int, cmp_stride: int, Q, K, valid_len, score_scale: float = 0.0,
                     sel_pos=None, ws=None, stream=None):
    """blossom_select_positions: the printed selection rule, one row per position and key/value group.
    p.block is the selection block size, p.topk is k.  Returns sel_pos int32 [B,G,L,topk]."""
    rc = (_fast or fastcall()).select_positions(p, kv_groups, cmp_block, cmp_stride, Q, K, valid_len, score_scale, sel_pos, ws,
                                                stream)
    if rc is not None:
        if rc:
            raise BlossomError(rc, "blossom_select_positions")
        return sel_pos
    import torch
    dt = _torch_dtype(p)
    _check_tensor(Q, (p.B, p.H, p.L, p.d), dt, "Q")
    _check_tensor(K, (p.B, kv_groups, p.L, p.d), dt, "K")
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    if sel_pos is None:
        sel_pos = torch.empty((p.B, kv_groups, p.L, p.topk), dtype=torch.int32, device=Q.device)
    _check_tensor(sel_pos, (p.B, kv_groups, p.L, p.topk), torch.int32, "sel_pos")
    cp = p.c()
    need = select_positions_workspace_bytes(p, kv_groups, cmp_block, cmp_stride)
    if ws is None:
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=Q.device)
    nbytes = _ws_bytes(ws, need)
    rc = lib().blossom_select_positions(ctypes.byref(cp), kv_groups, cmp_block, cmp_stride, float(score_scale), _ptr(Q),
                                        _ptr(K), _ptr(valid_len), _ptr(sel_pos), _ptr(ws), nbytes, _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_select_positions")
    return sel_pos


def attn_fwd_positions(p: Params, kv_groups: int, Q, K, V, valid_len, sel_pos, gate_w, gate_b=None, out: FwdOut | None = None,
                       want_branches: bool = False, stream=None) -> FwdOut:
    """blossom_attn_fwd_positions: forward under one selection row per query position and key/value group
    (K, V [B,G,L,d], sel_pos [B,G,L,topk]).  `want_branches` also returns o_lt, o_st, lse_lt, lse_st."""
    if out is not None:
        rc = (_fast or fastcall()).attn_fwd_positions(p, kv_groups, Q, K, V, valid_len, sel_pos, gate_w, gate_b, out.O, out.o_lt,
                                                      out.o_st, out.lse_lt, out.lse_st, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_attn_fwd_positions")
            return out
    import torch
    shp = (p.B, p.H, p.L, p.d)
    dt = _torch_dtype(p)
    _check_tensor(Q, shp, dt, "Q")
    for t, nm in ((K, "K"), (V, "V")):
        _check_tensor(t, (p.B, kv_groups, p.L, p.d), dt, nm)
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    _check_tensor(sel_pos, (p.B, kv_groups, p.L, p.topk), torch.int32, "sel_pos")
    _check_tensor(gate_w, (p.H, 2 * p.d), torch.float32, "gate_w")
    _check_tensor(gate_b, (p.H,), torch.float32, "gate_b")
    if out is None:
        out = FwdOut(torch.empty(shp, dtype=dt, device=Q.device))
        if want_branches:
            out.o_lt = torch.empty(shp, dtype=torch.float32, device=Q.device)
            out.o_st = torch.empty(shp, dtype=torch.float32, device=Q.device)
            out.lse_lt = torch.empty(shp[:3], dtype=torch.float32, device=Q.device)
            out.lse_st = torch.empty(shp[:3], dtype=torch.float32, device=Q.device)
    cp = p.c()
    rc = lib().blossom_attn_fwd_positions(ctypes.byref(cp), kv_groups, _ptr(Q), _ptr(K), _ptr(V), _ptr(valid_len), _ptr(sel_pos),
                                          _ptr(gate_w), _ptr(gate_b), _ptr(out.O), _ptr(out.o_lt), _ptr(out.o_st),
                                          _ptr(out.lse_lt), _ptr(out.lse_st), _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_attn_fwd_positions")
    return out


def attn_bwd_positions(p: Params, kv_groups: int, Q, K, V, valid_len, sel_pos, gate_w, gate_b, fwd: FwdOut, dO,
                       out: BwdOut | None = None, ws=None, stream=None) -> BwdOut:
    """blossom_attn_bwd_positions: backward of attn_fwd_positions (dQ [B,H,L,d]; dK, dV [B,G,L,d]: the
    gradients of the query heads of a group added up)."""
    if out is not None:
        rc = (_fast or fastcall()).attn_bwd_positions(p, kv_groups, Q, K, V, valid_len, sel_pos, gate_w, gate_b, fwd.o_lt,
                                                      fwd.o_st, fwd.lse_lt, fwd.lse_st, dO, out.dQ, out.dK, out.dV,
                                                      out.d_gate_w, out.d_gate_b, ws, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_attn_bwd_positions")
            return out
    import torch
    shp = (p.B, p.H, p.L, p.d)
    kv_shp = (p.B, kv_groups, p.L, p.d)
    dt = _torch_dtype(p)
    for t, nm, sh in ((Q, "Q", shp), (K, "K", kv_shp), (V, "V", kv_shp), (dO, "dO", shp)):
        if t is None:
            raise ValueError(f"{nm} is required")
        _check_tensor(t, sh, dt, nm)
    for t, nm in ((fwd.o_lt, "o_lt"), (fwd.o_st, "o_st")):
        if t is None:
            raise ValueError(f"{nm} is required")
        _check_tensor(t, shp, torch.float32, nm)
    for t, nm in ((fwd.lse_lt, "lse_lt"), (fwd.lse_st, "lse_st")):
        if t is None:
            raise ValueError(f"{nm} is required")
        _check_tensor(t, shp[:3], torch.float32, nm)
    _check_tensor(valid_len, (p.B,), torch.int32, "valid_len")
    _check_tensor(sel_pos, (p.B, kv_groups, p.L, p.topk), torch.int32, "sel_pos")
    _check_tensor(gate_w, (p.H, 2 * p.d), torch.float32, "gate_w")
    _check_tensor(gate_b, (p.H,), torch.float32, "gate_b")
    if out is None:
        out = BwdOut(torch.empty(shp, dtype=dt, device=Q.device), torch.empty(kv_shp, dtype=dt, device=Q.device),
                     torch.empty(kv_shp, dtype=dt, device=Q.device),
                     torch.empty((p.H, 2 * p.d), dtype=torch.float32, device=Q.device),
                     torch.empty((p.H,), dtype=torch.float32, device=Q.device))
    _check_tensor(out.dQ, shp, dt, "dQ")
    _check_tensor(out.dK, kv_shp, dt, "dK")
    _check_tensor(out.dV, kv_shp, dt, "dV")
    _check_tensor(out.d_gate_w, (p.H, 2 * p.d), torch.float32, "d_gate_w")
    _check_tensor(out.d_gate_b, (p.H,), torch.float32, "d_gate_b")
    ws, nbytes = _workspace(p, WS_BWD, ws, Q.device)
    cp = p.c()
    rc = lib().blossom_attn_bwd_positions(ctypes.byref(cp), kv_groups, _ptr(Q), _ptr(K), _ptr(V), _ptr(valid_len),
                                          _ptr(sel_pos), _ptr(gate_w), _ptr(gate_b), _ptr(fwd.o_lt), _ptr(fwd.o_st),
                                          _ptr(fwd.lse_lt), _ptr(fwd.lse_st), _ptr(dO), _ptr(out.dQ), _ptr(out.dK),
                                          _ptr(out.dV), _ptr(out.d_gate_w), _ptr(out.d_gate_b), _ptr(ws), nbytes,
                                          _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_attn_bwd_positions")
    return out


def out_proj_ln(p: Params, d_model: int, O, W_O_t, H_prev, ln_gamma, ln_beta, ln_eps: float, bias=None, S=None,
                want_stats: bool = False, stream=None):
    """blossom_out_proj_ln: S = LayerNorm(H_prev + Concat_h(O[:, h]) W^O (+ bias)); W_O_t is [d_model, H*d].
    Returns S, or (S, mean, rstd) with want_stats."""
    import torch
    mean = rstd = None
    if want_stats:
        mean = torch.empty((p.B, p.L), dtype=torch.float32, device=O.device)
        rstd = torch.empty((p.B, p.L), dtype=torch.float32, device=O.device)
    if S is not None:
        rc = (_fast or fastcall()).out_proj_ln(p, d_model, O, W_O_t, bias, H_prev, ln_gamma, ln_beta, ln_eps, S, mean, rstd,
                                               stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_out_proj_ln")
            return (S, mean, rstd) if want_stats else S
    dt = _torch_dtype(p)
    _check_tensor(O, (p.B, p.H, p.L, p.d), dt, "O")
    _check_tensor(W_O_t, (d_model, p.H * p.d), dt, "W_O_t")
    _check_tensor(H_prev, (p.B, p.L, d_model), dt, "H_prev")
    _check_tensor(ln_gamma, (d_model,), torch.float32, "ln_gamma")
    _check_tensor(ln_beta, (d_model,), torch.float32, "ln_beta")
    _check_tensor(bias, (d_model,), torch.float32, "bias")
    if S is None:
        S = torch.empty((p.B, p.L, d_model), dtype=dt, device=O.device)
    _check_tensor(S, (p.B, p.L, d_model), dt, "S")
    cp = p.c()
    rc = lib().blossom_out_proj_ln(ctypes.byref(cp), d_model, _ptr(O), _ptr(W_O_t), _ptr(bias), _ptr(H_prev), _ptr(ln_gamma),
                                   _ptr(ln_beta), float(ln_eps), _ptr(S), _ptr(mean), _ptr(rstd), _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_out_proj_ln")
    return (S, mean, rstd) if want_stats else S


@dataclass
class PagedParams:
    """blossom_paged_params: a batch of S sequences in a paged key/value cache, bringing T new tokens together."""
    S: int
    T: int
    H: int
    G: int
    d: int
    page: int
    n_pages: int
    max_pages: int
    dtype: int = F32
    softmax_scale: float = 0.0
    window: int = 0
    max_len: int = 0
    table_per_head: int = 0

    def c(self) -> BlossomPagedParams:
        return BlossomPagedParams(self.S, self.T, self.H, self.G, self.d, self.page, self.n_pages, self.max_pages, self.dtype,
                                  self.softmax_scale, self.window, self.max_len, self.table_per_head)

    @property
    def capacity(self) -> int:
        """Positions that a sequence may hold: rows of the rotary tables."""
        held = self.max_pages * self.page
        return min(self.max_len, held) if self.max_len > 0 else held


def paged_workspace_bytes(p: PagedParams, which: int) -> int:
    cp = p.c()
    return int(lib().blossom_paged_workspace_bytes(ctypes.byref(cp), which))


def _token_stride(t, rows, heads, d, dtype, name) -> int:
    """Elements from a token's row to the next of a [rows, heads, d] tensor whose heads and channels are contiguous."""
    if t is None:
        raise ValueError(f"{name} is required")
    if tuple(t.shape) != (rows, heads, d) or t.dtype != dtype or not t.is_cuda or t.stride(2) != 1 or (heads > 1 and t.stride(1) != d):
        raise ValueError(f"{name}: expected cuda tensor {(rows, heads, d)} {dtype} with contiguous heads and channels, got "
                         f"{tuple(t.shape)} {t.dtype} strides={tuple(t.stride())} cuda={t.is_cuda}")
    if rows > 1 and t.stride(0) < heads * d:  # (an expanded tensor's 0 would mean rows one after another)
        raise ValueError(f"{name}: expected tokens that do not overlap, got a token stride of {t.stride(0)} for rows of {heads * d}")
    return t.stride(0) if rows > 1 else 0


def _check_cache(p: PagedParams, K_cache, V_cache, page_table, cu_seqlens, kv_len):
    import torch
    for t, nm in ((K_cache, "K_cache"), (V_cache, "V_cache"), (page_table, "page_table"), (kv_len, "kv_len")):
        if t is None:
            raise ValueError(f"{nm} is required")
    shp = (p.n_pages, p.G, p.page, p.d)
    _check_tensor(K_cache, shp, _torch_dtype(p), "K_cache")
    _check_tensor(V_cache, shp, _torch_dtype(p), "V_cache")
    _check_tensor(page_table, (p.S, p.G, p.max_pages) if p.table_per_head else (p.S, p.max_pages), torch.int32, "page_table")
    _check_tensor(cu_seqlens, (p.S + 1,), torch.int32, "cu_seqlens")
    _check_tensor(kv_len, (p.S,), torch.int32, "kv_len")


def _on(stream):
    """For buffers that a call on `stream` needs: the allocator gives their memory on to that stream's work alone, and not to the
    current stream's while the call still runs."""
    import contextlib
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def kv_append(p: PagedParams, K, V, K_cache, V_cache, page_table, cu_seqlens, kv_len, Q=None, rope=None, Q_rot=None, stream=None):
    """blossom_kv_append: the new tokens' K and V [T,G,d] go into the cache, K rotated with rope=(cos, sin).  Returns Q_rot
    [T,H,d], the rotated Q (None without Q).  K, V and Q may be slices of one projection: a token's heads are contiguous.
    What the call allocates belongs to `stream` (the current one if None): memory used elsewhere is the caller's to hold."""
    cos, sin = rope if rope is not None else (None, None)
    if Q is None or Q_rot is not None:
        rc = (_fast or fastcall()).kv_append(p, Q, K, V, cos, sin, page_table, cu_seqlens, kv_len, K_cache, V_cache, Q_rot, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_kv_append")
            return Q_rot
    return _append(p, "blossom_kv_append", K, V, K_cache, V_cache, page_table, cu_seqlens, kv_len, None, Q, cos, sin, Q_rot, stream)


def _append(p: PagedParams, name, K, V, K_cache, V_cache, page_table, cu_seqlens, kv_len, tree_mask, Q, cos, sin, Q_rot, stream):
    """The Python path of kv_append and kv_append_tree: allocates what is missing, names what is wrong."""
    import torch
    dt = _torch_dtype(p)
    ks, vs = _token_stride(K, p.T, p.G, p.d, dt, "K"), _token_stride(V, p.T, p.G, p.d, dt, "V")
    qs = 0
    if Q is not None:
        qs = _token_stride(Q, p.T, p.H, p.d, dt, "Q")
        if Q_rot is None:
            with _on(stream):
                Q_rot = torch.empty((p.T, p.H, p.d), dtype=dt, device=Q.device)
    _check_tensor(Q_rot, (p.T, p.H, p.d), dt, "Q_rot")
    if cu_seqlens is None:
        raise ValueError("cu_seqlens is required")
    _check_cache(p, K_cache, V_cache, page_table, cu_seqlens, kv_len)
    _check_tensor(cos, (p.capacity, p.d // 2), torch.float32, "rope_cos")
    _check_tensor(sin, (p.capacity, p.d // 2), torch.float32, "rope_sin")
    _check_tensor(tree_mask, (p.T,), torch.int64, "tree_mask")
    cp = p.c()
    mask = () if tree_mask is None else (_ptr(tree_mask),)
    rc = getattr(lib(), name)(ctypes.byref(cp), _ptr(Q), qs, _ptr(K), ks, _ptr(V), vs, _ptr(cos), _ptr(sin), _ptr(page_table),
                              _ptr(cu_seqlens), _ptr(kv_len), *mask, _ptr(K_cache), _ptr(V_cache), _ptr(Q_rot), _stream(stream))
    if rc:
        raise BlossomError(rc, name)
    return Q_rot


def _paged_attn(p: PagedParams, which, rows, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, O, lse, ws, stream, tree_mask=None):
    """The Python path of attn_decode, attn_prompt and attn_tree: allocates what is missing, names what is wrong."""
    import torch
    dt = _torch_dtype(p)
    qs = _token_stride(Q, rows, p.H, p.d, dt, "Q")
    _check_cache(p, K_cache, V_cache, page_table, cu_seqlens, kv_len)
    need = paged_workspace_bytes(p, which)
    _ws_bytes(ws, need)
    with _on(stream):
        if O is None:
            O = torch.empty((rows, p.H, p.d), dtype=dt, device=Q.device)
        if ws is None and need > 0:
            ws = torch.empty(need, dtype=torch.uint8, device=Q.device)
    _check_tensor(O, (rows, p.H, p.d), dt, "O")
    _check_tensor(lse, (rows, p.H), torch.float32, "lse")
    nbytes = _ws_bytes(ws, need)
    cp = p.c()
    head = (ctypes.byref(cp), _ptr(Q), qs, _ptr(K_cache), _ptr(V_cache), _ptr(page_table))
    tail = (_ptr(kv_len), _ptr(O), _ptr(lse), _ptr(ws), nbytes, _stream(stream))
    if which == WS_DECODE:
        name, rc = "blossom_attn_decode", lib().blossom_attn_decode(*head, *tail)
    elif which == WS_TREE:
        name, rc = "blossom_attn_tree", lib().blossom_attn_tree(*head, _ptr(cu_seqlens), tail[0], _ptr(tree_mask), *tail[1:])
    else:
        name, rc = "blossom_attn_prompt", lib().blossom_attn_prompt(*head, _ptr(cu_seqlens), *tail)
    if rc:
        raise BlossomError(rc, name)
    return O, lse


def attn_decode(p: PagedParams, Q, K_cache, V_cache, page_table, kv_len, O=None, lse=None, ws=None, stream=None):
    """blossom_attn_decode: one new token a sequence (Q [S,H,d]) over its cached positions.  Returns (O, lse); lse is written
    where given."""
    if O is not None:
        rc = (_fast or fastcall()).attn_decode(p, Q, K_cache, V_cache, page_table, kv_len, O, lse, ws, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_attn_decode")
            return O, lse
    return _paged_attn(p, WS_DECODE, p.S, Q, K_cache, V_cache, page_table, None, kv_len, O, lse, ws, stream)


def attn_prompt(p: PagedParams, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, O=None, lse=None, ws=None, stream=None):
    """blossom_attn_prompt: causal attention of packed new tokens (Q [T,H,d]) over their sequences' cached positions, their own
    among them.  Returns (O, lse); lse is written where given."""
    if O is not None:
        rc = (_fast or fastcall()).attn_prompt(p, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, O, lse, ws, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_attn_prompt")
            return O, lse
    if cu_seqlens is None:
        raise ValueError("cu_seqlens is required")
    return _paged_attn(p, WS_PROMPT, p.T, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, O, lse, ws, stream)


_MOST = 2**31 - 1  # of what the library counts in 32 bits


def _here(**tensors):
    """All of them on the current device, whose stream the call goes to."""
    import torch
    now = torch.cuda.current_device() if torch.cuda.is_initialized() else 0
    for name, t in tensors.items():
        if t is not None and (not t.is_cuda or (t.device.index or 0) != now):
            raise ValueError(f"{name}: expected a tensor on the current device, cuda:{now}, got one on {t.device}")


def kv_append_tree(p: PagedParams, K, V, K_cache, V_cache, page_table, cu_seqlens, kv_len, tree_mask, Q=None, rope=None, Q_rot=None,
                   stream=None):
    """blossom_kv_append_tree: kv_append for drafted tokens, each rotated by its position in its tree.  tree_mask int64 [T]: bit k of
    a token's says that it sees drafted token k of its sequence.  Returns Q_rot."""
    cos, sin = rope if rope is not None else (None, None)
    if Q is None or Q_rot is not None:
        rc = (_fast or fastcall()).kv_append_tree(p, Q, K, V, cos, sin, page_table, cu_seqlens, kv_len, tree_mask, K_cache, V_cache,
                                                  Q_rot, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_kv_append_tree")
            return Q_rot
    if tree_mask is None:
        raise ValueError("tree_mask is required")
    _here(K=K, V=V, K_cache=K_cache, V_cache=V_cache, page_table=page_table, cu_seqlens=cu_seqlens, kv_len=kv_len, tree_mask=tree_mask,
          Q=Q, rope_cos=cos, rope_sin=sin, Q_rot=Q_rot)
    return _append(p, "blossom_kv_append_tree", K, V, K_cache, V_cache, page_table, cu_seqlens, kv_len, tree_mask, Q, cos, sin, Q_rot,
                   stream)


def attn_tree(p: PagedParams, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, tree_mask, O=None, lse=None, ws=None, stream=None):
    """blossom_attn_tree: attention of drafted tokens (Q [T,H,d]) over their sequences' histories and the drafted tokens that
    tree_mask (int64 [T]) names.  Returns (O, lse); lse is written where given."""
    if O is not None:
        rc = (_fast or fastcall()).attn_tree(p, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, tree_mask, O, lse, ws, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_attn_tree")
            return O, lse
    import torch
    if cu_seqlens is None:
        raise ValueError("cu_seqlens is required")
    if tree_mask is None:
        raise ValueError("tree_mask is required")
    _check_tensor(tree_mask, (p.T,), torch.int64, "tree_mask")
    _here(Q=Q, K_cache=K_cache, V_cache=V_cache, page_table=page_table, cu_seqlens=cu_seqlens, kv_len=kv_len, tree_mask=tree_mask, O=O,
          lse=lse, ws=ws)
    return _paged_attn(p, WS_TREE, p.T, Q, K_cache, V_cache, page_table, cu_seqlens, kv_len, O, lse, ws, stream, tree_mask)


def kv_accept(p: PagedParams, keep, K_cache, V_cache, page_table, cu_seqlens, kv_len, new_len=None, stream=None):
    """blossom_kv_accept: of each sequence's drafted tokens those that keep (int32 [S, n], ascending, then -1) lists move down behind the
    history.  Returns new_len int32 [S], the lengths then; kv_len stays, for the other layers' calls."""
    if new_len is not None:
        rc = (_fast or fastcall()).kv_accept(p, keep, K_cache, V_cache, page_table, cu_seqlens, kv_len, new_len, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_kv_accept")
            return new_len
    import torch
    if keep is None or cu_seqlens is None:
        raise ValueError("keep and cu_seqlens are required")
    if keep.dim() != 2 or keep.shape[0] != p.S or not 1 <= keep.shape[1] <= _MOST:
        raise ValueError(f"keep: expected shape ({p.S}, 1 <= n <= {_MOST}), got {tuple(keep.shape)}")
    _check_tensor(keep, keep.shape, torch.int32, "keep")
    _check_cache(p, K_cache, V_cache, page_table, cu_seqlens, kv_len)
    _here(keep=keep, K_cache=K_cache, V_cache=V_cache, page_table=page_table, cu_seqlens=cu_seqlens, kv_len=kv_len, new_len=new_len)
    if new_len is None:
        with _on(stream):
            new_len = torch.empty(p.S, dtype=torch.int32, device=keep.device)
    _check_tensor(new_len, (p.S,), torch.int32, "new_len")
    cp = p.c()
    rc = lib().blossom_kv_accept(ctypes.byref(cp), keep.shape[1], _ptr(keep), _ptr(page_table), _ptr(cu_seqlens), _ptr(kv_len),
                                 _ptr(K_cache), _ptr(V_cache), _ptr(new_len), _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_kv_accept")
    return new_len


def fork_workspace_bytes(p: PagedParams, n_new: int) -> int:
    cp = p.c()
    return int(lib().blossom_fork_workspace_bytes(ctypes.byref(cp), n_new))


def kv_fork(p: PagedParams, parent, page_table, kv_len, refs, grow=0, new_table=None, new_len=None, new_refs=None, copies=None,
            missing=None, ws=None, stream=None):
    """blossom_kv_fork: parent int32 [N] says which of p.S sequences each of N new ones goes on from, with room for `grow` more
    positions.  Returns (new_table [N, max_pages], new_len [N], new_refs [n_pages], copies [N, 3], missing [1]): whole pages are shared,
    `copies` goes to kv_copy_pages for each layer, `missing` counts the pages that there were not."""
    if new_table is not None:
        rc = (_fast or fastcall()).kv_fork(p, parent, page_table, kv_len, refs, grow, new_table, new_len, new_refs, copies, missing, ws,
                                           stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_kv_fork")
            return new_table, new_len, new_refs, copies, missing
    import torch
    for t, nm in ((parent, "parent"), (page_table, "page_table"), (kv_len, "kv_len"), (refs, "refs")):
        if t is None:
            raise ValueError(f"{nm} is required")
    if parent.dim() != 1 or not 1 <= parent.shape[0] <= _MOST:
        raise ValueError(f"parent: expected shape (1 <= n <= {_MOST},), got {tuple(parent.shape)}")
    if not -_MOST <= grow <= _MOST:
        raise ValueError(f"grow: expected 32 bits, got {grow}")
    N, i32 = parent.shape[0], torch.int32
    _check_tensor(parent, (N,), i32, "parent")
    _check_tensor(page_table, (p.S, p.max_pages), i32, "page_table")
    _check_tensor(kv_len, (p.S,), i32, "kv_len")
    _check_tensor(refs, (p.n_pages,), i32, "refs")
    _here(parent=parent, page_table=page_table, kv_len=kv_len, refs=refs, new_table=new_table, new_len=new_len, new_refs=new_refs,
          copies=copies, missing=missing, ws=ws)
    need = fork_workspace_bytes(p, N)
    shapes = ((new_table, (N, p.max_pages), "new_table"), (new_len, (N,), "new_len"), (new_refs, (p.n_pages,), "new_refs"),
              (copies, (N, 3), "copies"), (missing, (1,), "missing"))
    with _on(stream):
        out = [torch.empty(shape, dtype=i32, device=parent.device) if t is None else t for t, shape, _ in shapes]
        if ws is None:
            ws = torch.empty(max(need, 16), dtype=torch.uint8, device=parent.device)
    for t, (_, shape, nm) in zip(out, shapes):
        _check_tensor(t, shape, i32, nm)
    nbytes = _ws_bytes(ws, need)
    cp = p.c()
    rc = lib().blossom_kv_fork(ctypes.byref(cp), N, grow, _ptr(parent), _ptr(page_table), _ptr(kv_len), _ptr(refs), *map(_ptr, out),
                               _ptr(ws), nbytes, _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_kv_fork")
    return tuple(out)


def kv_copy_pages(p: PagedParams, copies, K_cache, V_cache, stream=None):
    """blossom_kv_copy_pages: copies int32 [N, 3] of (source page, target page, positions) in both caches of a layer."""
    rc = (_fast or fastcall()).kv_copy_pages(p, copies, K_cache, V_cache, stream)
    if rc is not None:
        if rc:
            raise BlossomError(rc, "blossom_kv_copy_pages")
        return
    import torch
    for t, nm in ((copies, "copies"), (K_cache, "K_cache"), (V_cache, "V_cache")):
        if t is None:
            raise ValueError(f"{nm} is required")
    if copies.dim() != 2 or not 1 <= copies.shape[0] <= _MOST or copies.shape[1] != 3:
        raise ValueError(f"copies: expected shape (1 <= n <= {_MOST}, 3), got {tuple(copies.shape)}")
    _check_tensor(copies, copies.shape, torch.int32, "copies")
    shp = (p.n_pages, p.G, p.page, p.d)
    _check_tensor(K_cache, shp, _torch_dtype(p), "K_cache")
    _check_tensor(V_cache, shp, _torch_dtype(p), "V_cache")
    _here(copies=copies, K_cache=K_cache, V_cache=V_cache)
    cp = p.c()
    rc = lib().blossom_kv_copy_pages(ctypes.byref(cp), copies.shape[0], _ptr(copies), _ptr(K_cache), _ptr(V_cache), _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_kv_copy_pages")


@dataclass
class BeamParams:
    """blossom_beam_params: B histories of W beams each, of whose continuations by any of V items the K best are chosen."""
    B: int
    W: int
    K: int
    V: int
    dtype: int = F32
    eos: int = -1

    def c(self) -> BlossomBeamParams:
        return BlossomBeamParams(self.B, self.W, self.K, self.V, self.dtype, self.eos)


def beam_workspace_bytes(p: BeamParams) -> int:
    cp = p.c()
    return int(lib().blossom_beam_workspace_bytes(ctypes.byref(cp)))


def beam_select(p: BeamParams, logits, score, ended=None, parent=None, token=None, out_score=None, out_ended=None, ws=None, stream=None):
    """blossom_beam_select: logits [B*W, V] (rows may be slices of wider ones), score fp32 [B, W], ended bool or uint8 [B, W] or None.
    Returns (parent, token, out_score, out_ended), each [B, K], the best first: parent is a row of `logits`."""
    if parent is not None and out_ended is not None:
        rc = (_fast or fastcall()).beam_select(p, logits, score, ended, parent, token, out_score, out_ended, ws, stream)
        if rc is not None:
            if rc:
                raise BlossomError(rc, "blossom_beam_select")
            return parent, token, out_score, out_ended
    import torch
    if logits is None or score is None:
        raise ValueError("logits and score are required")
    rows = p.B * p.W
    if tuple(logits.shape) != (rows, p.V) or logits.dtype != _torch_dtype(p) or not logits.is_cuda or (p.V > 1 and logits.stride(1) != 1) or \
            (rows > 1 and logits.stride(0) < p.V):
        raise ValueError(f"logits: expected cuda tensor {(rows, p.V)} {_torch_dtype(p)} of contiguous rows that do not overlap, got "
                         f"{tuple(logits.shape)} {logits.dtype} strides={tuple(logits.stride())} cuda={logits.is_cuda}")
    _check_tensor(score, (p.B, p.W), torch.float32, "score")
    flags = (torch.bool, torch.uint8)
    _check_tensor(ended, (p.B, p.W), ended.dtype if ended is not None and ended.dtype in flags else torch.bool, "ended")
    _here(logits=logits, score=score, ended=ended, parent=parent, token=token, out_score=out_score, out_ended=out_ended, ws=ws)
    need = beam_workspace_bytes(p)
    with _on(stream):
        def new(t, dtype):
            return torch.empty((p.B, p.K), dtype=dtype, device=logits.device) if t is None else t

        parent, token, out_score, out_ended = new(parent, torch.int32), new(token, torch.int32), new(out_score, torch.float32), new(out_ended, torch.bool)
        if ws is None:
            ws = torch.empty(max(need, 16), dtype=torch.uint8, device=logits.device)
    _check_tensor(parent, (p.B, p.K), torch.int32, "parent")
    _check_tensor(token, (p.B, p.K), torch.int32, "token")
    _check_tensor(out_score, (p.B, p.K), torch.float32, "out_score")
    _check_tensor(out_ended, (p.B, p.K), out_ended.dtype if out_ended.dtype in flags else torch.bool, "out_ended")
    nbytes = _ws_bytes(ws, need)
    cp = p.c()
    rc = lib().blossom_beam_select(ctypes.byref(cp), _ptr(logits), logits.stride(0) if rows > 1 else 0, _ptr(score), _ptr(ended), _ptr(parent),
                                   _ptr(token), _ptr(out_score), _ptr(out_ended), _ptr(ws), nbytes, _stream(stream))
    if rc:
        raise BlossomError(rc, "blossom_beam_select")
    return parent, token, out_score, out_ended
