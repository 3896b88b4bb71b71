#!/usr/bin/env python3
"""Benchmark of the Blossom attention hot path on one MI355X.

One step = one pass of the whole path over one batch of seeded synthetic input that is
already resident in HBM: block selection, fused forward (saving what backward needs) and
backward.  The headline value is valid tokens per second of that step.  The same JSON line
carries the stage times, the forward-only rate (the quantity the L=8192 target is stated
on), a roofline object for the dominant kernel, the same-style dense causal kernel and the
CPU oracle timed on a bounded sample of the same workload.

The default run (workload cfg4, L=8192) also times the L=1024 training step (cfg5) and the paper's own
short-sequence shape (cfg2, L=200, fp32) the same way and reports them under "l1024_training_step" and
"l200_training_step".  Roofline entries count algorithmic work only: forward 4d
flops per unmasked pair, the whole backward 10d (five contractions), bytes of valid positions.
"out_proj_ln" times the layer around the attention (output projection + residual + LayerNorm in one
kernel, every position) on the forward's output buffer; it is not part of the step.

    python bench.py [--gpus 1] [--steps K] [--warmup W] [--workload cfg4]
    python bench.py --stage <kernel>        one stage alone (for profilers)
    python bench.py --stage ceiling         stripped tile loop of the forward: what the pipes allow
    python bench.py --stage positions       the path under the selection rule as printed, at the paper's own setting
"""
from __future__ import annotations

import argparse
import json
import os
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np

PROFILES = os.path.join(ROOT, "profiles")
CSRC = os.path.join(ROOT, "paper_2512_13368_amd", "csrc")


def sources_sha256():
    """Hash of the kernel sources that the workloads run (the paged cache's and beam search's serve no workload here): a
    stored profile figure is only quoted for the code it was measured on."""
    import hashlib
    h = hashlib.sha256()
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".hip", ".h")) and not name.startswith(("paged", "beam")):
            h.update(name.encode())
            h.update(open(os.path.join(CSRC, name), "rb").read())
    return h.hexdigest()


def profiled_traffic(workload):
    """HBM-side bytes per launch from profiles/<workload>_hbm_traffic.txt (rocprofv3 --pmc FETCH_SIZE /
    WRITE_SIZE, scaled by a plain copy of known size; the file gives the commands).  The file names the
    hash of the kernel sources it was measured on; for any other sources nothing is quoted (None)."""
    path = os.path.join(PROFILES, f"{workload}_hbm_traffic.txt")
    if not os.path.exists(path):
        return {}, None
    table, sha = {}, None
    for line in open(path):
        t = line.split()
        if len(t) == 3 and t[0] == "traffic_bytes":
            table[t[1]] = int(t[2])
        elif len(t) == 2 and t[0] == "sources_sha256":
            sha = t[1]
    if sha != sources_sha256():
        return {}, sha
    return table, sha


HBM_PEAK_GBS = 8000.0          # MI355X HBM3E
MFMA_BF16_PEAK_TFLOPS = 2500.0  # dense bf16 MFMA
FP32_VALU_PEAK_TFLOPS = 157.3   # 256 CU x 4 SIMD x 64 FLOP/clk x 2.4 GHz


def algorithmic_pairs(w, valid_len, sel):
    """Unmasked (query, key) pairs of the two branches, from the selection lists (integer
    bookkeeping only; no attention arithmetic)."""
    L, b, win, NB = w.L, w.block, w.window, w.NB
    lt = st = dense = 0
    blk_lo = np.arange(NB) * b
    blk_hi = np.minimum(blk_lo + b, L)
    for r in range(w.B):
        n = int(valid_len[r])
        p0 = L - n
        if n == 0:
            continue
        i = np.arange(p0, L)
        if w.stis_block == 0:
            st += int(np.minimum(win, i - p0 + 1).sum()) * w.H
        else:
            # all of Eq. 15, causal: the window and the last-block term are suffixes of [p0, i]; the
            # blocks at power-of-two block distances lie below them and are disjoint
            sb = w.stis_block
            lo = np.maximum(p0, i - win + 1)
            lo = np.where(i >= L - sb, np.minimum(lo, max(p0, L - sb)), lo)
            cnt = i - lo + 1
            bq = i // sb
            e2 = 0
            while (1 << e2) <= int(bq.max()):
                bk = bq - (1 << e2)
                k_lo = np.maximum(bk * sb, p0)
                k_hi = np.minimum(np.minimum((bk + 1) * sb - 1, L - 1), lo - 1)
                cnt = cnt + np.where(bk >= 0, np.clip(k_hi - k_lo + 1, 0, None), 0)
                e2 += 1
            st += int(cnt.sum()) * w.H
        dense += n * (n + 1) // 2 * w.H
        vcount = np.clip(blk_hi - np.maximum(blk_lo, p0), 0, None)          # valid positions per block
        first = np.maximum(blk_lo, p0)
        diag = vcount * (vcount + 1) // 2                                    # causal pairs inside a block
        s = sel[r]                                                           # [H,NB,k]
        mask = s >= 0
        I = np.broadcast_to(np.arange(NB)[None, :, None], s.shape)
        off = mask & (s != I)
        kv = np.where(off, vcount[np.clip(s, 0, NB - 1)], 0).sum(-1)         # keys in selected past blocks
        has_diag = (mask & (s == I)).any(-1)
        lt += int((kv * vcount[None, :]).sum() + (has_diag * diag[None, :]).sum())
        del first
    return lt, st, dense


STAGES = ["select", "rope_select", "fwd", "fwd_save", "bwd", "bwd_gate", "bwd_inverse", "bwd_dq", "bwd_dkv", "bwd_dq_dkv", "dense", "serve", "copy",
          "out_proj"]
PROBE_KINDS = ["matrix instructions only", "softmax VALU work only", "both, operands in registers",
               "both, operands from LDS", "whole tile loop (with global->LDS staging)", "staging only"]


class Runner:
    """Device buffers and launch closures of one workload (everything allocated once, up front)."""

    def __init__(self, w, n_sets, torch, B, make_inputs, bf16_bits):
        self.w, self.torch, self.B = w, torch, B
        dev = torch.device("cuda:0")
        self.xs = [make_inputs(w, input_set=i, want_dO=True) for i in range(n_sets)]
        self.x = self.xs[0]  # the per-kernel passes, the pair counts and the CPU baseline use the first set

        def up(a):
            if w.dtype == "bf16":
                return torch.from_numpy(bf16_bits(a).view(np.int16)).to(dev).view(torch.bfloat16)
            return torch.from_numpy(a).to(dev)

        self.sets = [(up(xi.Q), up(xi.K), up(xi.V), up(xi.dO), torch.from_numpy(xi.valid_len).to(dev)) for xi in self.xs]
        self.gw = torch.from_numpy(self.x.gate_w).to(dev)
        self.gb = torch.from_numpy(self.x.gate_b).to(dev)
        dt = B.F32 if w.dtype == "fp32" else B.BF16
        stis = dict(stis_mode=int(w.stis_block > 0), stis_block=w.stis_block)
        mkp = lambda **kw: B.Params(w.B, w.H, w.L, w.d, w.block, w.topk, w.window, dt, **stis, **kw)
        self.p, self.p_nosave, self.p_serve = mkp(save_for_bwd=1), mkp(), mkp(last_block_only=1)
        tdt = torch.float32 if w.dtype == "fp32" else torch.bfloat16
        shp = (w.B, w.H, w.L, w.d)
        mk = lambda: torch.empty(shp, dtype=tdt, device=dev)
        mk32 = lambda: torch.empty(shp, dtype=torch.float32, device=dev)
        self.sel = torch.empty((w.B, w.H, w.NB, w.topk), dtype=torch.int32, device=dev)
        self.fo = B.FwdOut(mk(), mk32(), mk32(), torch.empty(shp[:3], dtype=torch.float32, device=dev),
                           torch.empty(shp[:3], dtype=torch.float32, device=dev))
        self.fo_nosave = B.FwdOut(self.fo.O)
        self.bo = B.BwdOut(mk(), mk(), mk(), torch.empty((w.H, 2 * w.d), dtype=torch.float32, device=dev),
                           torch.empty((w.H,), dtype=torch.float32, device=dev))
        self.ws_sel = torch.empty(max(1, B.workspace_bytes(self.p, B.WS_SELECT)), dtype=torch.uint8, device=dev)
        self.ws_bwd = torch.empty(max(1, B.workspace_bytes(self.p, B.WS_BWD)), dtype=torch.uint8, device=dev)
        self.ws_fwd = torch.empty(max(1, B.workspace_bytes(self.p, B.WS_FWD)), dtype=torch.uint8, device=dev)
        self.O_dense = mk()

    def step(self, i=0):
        B, p = self.B, self.p
        Q, K, V, dO, vl = self.sets[i % len(self.sets)]
        B.select_blocks(p, Q, K, vl, sel=self.sel, ws=self.ws_sel)
        B.attn_fwd(p, Q, K, V, vl, self.sel, self.gw, self.gb, out=self.fo, ws=self.ws_fwd)
        B.attn_bwd(p, Q, K, V, vl, self.sel, self.gw, self.gb, self.fo, dO, out=self.bo, ws=self.ws_bwd)

    def stage_fn(self, name):
        B, p = self.B, self.p
        Q, K, V, dO, vl = self.sets[0]
        sel, gw, gb, fo = self.sel, self.gw, self.gb, self.fo
        bwd = lambda st: (lambda: B.attn_bwd(p, Q, K, V, vl, sel, gw, gb, fo, dO, out=self.bo, ws=self.ws_bwd, stages=st))
        return {
            "select": lambda: B.select_blocks(p, Q, K, vl, sel=sel, ws=self.ws_sel),
            # selection with the rotary position embedding of Q and K fused into its pooling pass
            "rope_select": lambda: self._rope_select()(),
            "fwd": lambda: B.attn_fwd(self.p_nosave, Q, K, V, vl, sel, gw, gb, out=self.fo_nosave, ws=self.ws_fwd),
            "fwd_save": lambda: B.attn_fwd(p, Q, K, V, vl, sel, gw, gb, out=fo, ws=self.ws_fwd),
            "bwd": bwd(B.BWD_ALL), "bwd_gate": bwd(B.BWD_GATE), "bwd_inverse": bwd(B.BWD_INVERSE),
            "bwd_dq": bwd(B.BWD_DQ), "bwd_dkv": bwd(B.BWD_DKV),
            # dQ and dK/dV as the full call launches them (one grid on the matrix-core kernels)
            "bwd_dq_dkv": bwd(B.BWD_DQ | B.BWD_DKV),
            "dense": lambda: B.dense_causal_fwd(p, Q, K, V, vl, O=self.O_dense),
            # serving: selection and forward of the last query block only (the scored position)
            "serve": lambda: (B.select_blocks(self.p_serve, Q, K, vl, sel=sel, ws=self.ws_sel),
                              B.attn_fwd(self.p_serve, Q, K, V, vl, sel, gw, gb, out=self.fo_nosave, ws=self.ws_fwd)),
            # a plain device copy of one [B,H,L,d] tensor: calibrates the HBM byte counters
            "copy": lambda: self.O_dense.copy_(Q),
            # the layer around the attention: output projection + residual + LayerNorm on the forward's output
            "out_proj": lambda: self._out_proj()(),
        }[name]

    def _out_proj(self):
        if getattr(self, "_op_fn", None) is None:  # weights and buffers are made on first use, once
            torch, B, w = self.torch, self.B, self.w
            Q = self.sets[0][0]
            Dm = w.H * w.d
            g = torch.Generator(device="cpu").manual_seed(4242)
            Wt = (torch.randn((Dm, Dm), generator=g) / Dm ** 0.5).to(Q.dtype).to(Q.device)
            Hp = torch.randn((w.B, w.L, Dm), generator=g).to(Q.dtype).to(Q.device)
            gamma, beta = torch.ones(Dm, device=Q.device), torch.zeros(Dm, device=Q.device)
            S = torch.empty_like(Hp)
            self._op_fn = lambda: B.out_proj_ln(self.p, Dm, self.fo.O, Wt, Hp, gamma, beta, 1e-5, S=S)
        return self._op_fn

    def _rope_select(self):
        if getattr(self, "_rope_fn", None) is None:  # tables and output buffers are made on first use, once
            from paper_2512_13368_amd.inputs import rope_tables
            torch, B, w = self.torch, self.B, self.w
            Q, K, V, dO, vl = self.sets[0]
            cos, sin = (torch.from_numpy(t).to(Q.device) for t in rope_tables(w.L, w.d))
            Qr, Kr = torch.empty_like(Q), torch.empty_like(K)
            self._rope_fn = lambda: B.rope_select_blocks(self.p, Q, K, cos, sin, vl, Q_rot=Qr, K_rot=Kr, sel=self.sel,
                                                        ws=self.ws_sel)
        return self._rope_fn

    def timed(self, fn, reps):
        """Average launch time in ms with HIP events on the stream the work is launched on."""
        torch = self.torch
        ev0, ev1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        fn()
        torch.cuda.synchronize()
        ev0.record()
        for _ in range(reps):
            fn()
        ev1.record()
        torch.cuda.synchronize()
        return ev0.elapsed_time(ev1) / reps

    def kernel_times(self, reps, dense=True):
        ms = {k_: self.timed(self.stage_fn(s_), reps) for k_, s_ in (
            ("select", "select"), ("fwd", "fwd"), ("fwd_saving_for_bwd", "fwd_save"), ("bwd_gate", "bwd_gate"),
            ("bwd_inverse_list", "bwd_inverse"), ("bwd_dq", "bwd_dq"), ("bwd_dkv", "bwd_dkv"), ("bwd_dq_dkv", "bwd_dq_dkv"),
            ("bwd", "bwd"))}
        ms_dense = self.timed(self.stage_fn("dense"), max(2, reps // 4)) if dense else None
        return ms, ms_dense

    def work(self):
        """Algorithmic work per launch: unmasked pairs from the selection lists, bytes from the valid positions."""
        w = self.w
        nnz_lt, nnz_st, nnz_dense = algorithmic_pairs(w, self.x.valid_len, self.sel.cpu().numpy())
        pairs = nnz_lt + nnz_st
        sz = 4 if w.dtype == "fp32" else 2
        tensor = float(int(self.x.valid_len.sum())) * w.H * w.d   # elements of the valid positions of one tensor
        d = w.d
        # kernel -> (algorithmic flops, flops the kernel executes, bytes).  Forward: QK^T and PV (2d flops each per
        # unmasked pair).  Backward: five contractions per pair in all (S, dP, dV, dK, dQ = 10d flops, 2.5 x
        # forward); S and dP are needed by both backward kernels and recomputed in each, so each kernel is
        # charged half of them algorithmically (dQ: 2d + 2d, dK/dV: 4d + 2d) and executes 6d resp. 8d.
        # Bytes: every tensor a kernel has to read or write once, valid positions only.
        table = {
            "fwd": (4.0 * d * pairs, 4.0 * d * pairs, 4 * tensor * sz),                                   # Q,K,V | O
            "fwd_saving_for_bwd": (4.0 * d * pairs, 4.0 * d * pairs, 4 * tensor * sz + 2 * tensor * 4),   # + o_lt, o_st
            "bwd_dq": (4.0 * d * pairs, 6.0 * d * pairs, 5 * tensor * sz),                                # Q,K,V,dO | dQ
            "bwd_dkv": (6.0 * d * pairs, 8.0 * d * pairs, 6 * tensor * sz),                               # Q,K,V,dO | dK,dV
            # both in one launch, as the full backward call runs them: Q,K,V,dO read once, dQ,dK,dV written
            "bwd_dq_dkv": (10.0 * d * pairs, 14.0 * d * pairs, 7 * tensor * sz),
            "bwd_gate": (0.0, 0.0, tensor * (sz + 8)),                                                    # dO, o_lt, o_st
            "select": (0.0, 0.0, 2 * tensor * sz),                                                        # Q, K
            # the whole backward call: 10d flops per pair; Q,K,V,dO,o_lt,o_st read, dQ,dK,dV written
            "bwd": (10.0 * d * pairs, 14.0 * d * pairs, 7 * tensor * sz + 2 * tensor * 4),
        }
        return table, dict(nnz_lt=nnz_lt, nnz_st=nnz_st, nnz_dense=nnz_dense, pairs=pairs)


def roofline_entry(w, kernel, ms, table, traffic):
    flops, flops_exec, nbytes = table[kernel]
    mfma_peak = MFMA_BF16_PEAK_TFLOPS if w.dtype == "bf16" else FP32_VALU_PEAK_TFLOPS
    t = ms[kernel] * 1e-3
    if flops / (mfma_peak * 1e12) >= nbytes / (HBM_PEAK_GBS * 1e9):
        a = flops / t / 1e12
        r = {"bound": "mfma" if w.dtype == "bf16" else "alu", "achieved": round(a, 2), "peak": mfma_peak,
             "unit": "TFLOP/s", "frac": round(a / mfma_peak, 4)}
        if flops_exec != flops:
            r["frac_executed_incl_recompute"] = round(flops_exec / t / 1e12 / mfma_peak, 4)
    else:
        a = nbytes / t / 1e9
        r = {"bound": "hbm", "achieved": round(a, 1), "peak": HBM_PEAK_GBS, "unit": "GB/s",
             "frac": round(a / HBM_PEAK_GBS, 4)}
    r.update({"traffic": traffic.get(kernel), "kernel": kernel, "avg_launch_ms": round(ms[kernel], 4),
              "algorithmic_gflop": round(flops / 1e9, 2), "algorithmic_mb": round(nbytes / 1e6, 1)})
    return r


def measure_workload(w, args, mods, n_sets, headline):
    """Times the step and its kernels on workload w; returns the fields of the JSON line (headline) or a
    short summary (the second workload of the default run)."""
    torch, B, make_inputs, bf16_bits = mods
    R = Runner(w, n_sets, torch, B, make_inputs, bf16_bits)
    for i in range(args.warmup):
        R.step(i)
    torch.cuda.synchronize()
    run_step = R.step
    if args.graph and headline:
        # the library allocates nothing and never synchronises: the step is captured as it is
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            R.step()
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                R.step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        run_step = lambda i: graph.replay()
        run_step(0)
        torch.cuda.synchronize()

    # ---- timed region: exactly K steps ----
    t0 = time.perf_counter()
    for i in range(args.steps):
        run_step(i)
    torch.cuda.synchronize()
    wall = time.perf_counter() - t0
    ms_per_step = wall * 1e3 / args.steps

    reps = max(3, args.steps)
    ms, ms_dense = R.kernel_times(reps, dense=not args.no_dense)
    table, cnt = R.work()
    tokens = int(R.x.valid_len.sum())
    tokens_timed = sum(int(R.xs[i % n_sets].valid_len.sum()) for i in range(args.steps))  # over the timed steps
    traffic, traffic_sha = ({}, None) if (w.stis_block or args.shape) else profiled_traffic(w.name)
    roof = lambda k_: roofline_entry(w, k_, ms, table, traffic)
    # the launches of a step: on the bf16 matrix-core shapes a full backward call runs dQ and dK/dV as one kernel
    # (same condition as the library's dispatch).  The small-head kernels form the row constants in whichever pass runs and hold
    # the whole backward in one launch where a head fits LDS: a pass alone repeats the others' work, so theirs is taken as one.
    # Elsewhere dQ and dK/dV are two launches after the per-row pass.
    one_launch = w.dtype == "bf16" and w.d == 64 and w.block in (32, 64) and not w.bidir and \
        (w.stis_block == 0 or (w.stis_block <= w.block and w.stis_block & (w.stis_block - 1) == 0))
    small = w.d in (8, 16, 32) and w.block in (8, 16) and w.L <= 16384
    step_kernels = ["select", "fwd_saving_for_bwd"] + (["bwd"] if small else ["bwd_gate", "bwd_dq_dkv"] if one_launch
                                                       else ["bwd_gate", "bwd_dq", "bwd_dkv"])
    dominant = max(step_kernels, key=lambda k_: ms[k_])
    out = {
        "ms_per_step": round(ms_per_step, 4),
        "tokens_per_s": round(tokens_timed / wall, 1),
        "config": {"workload": f"{w.name}: B={w.B} H={w.H} L={w.L} d={w.d} b={w.block} k={w.topk} "
                               f"w={w.window} {w.dtype}, lens U[{w.len_lo},{w.len_hi}] left-padded, seed {w.seed}"
                               + (f", short-term mask = all of Eq. 15 with mask block {w.stis_block}" if w.stis_block else ""),
                   "tokens_per_step": tokens, "unmasked_pairs_lt": cnt["nnz_lt"], "unmasked_pairs_st": cnt["nnz_st"],
                   "launch": "hip graph replay" if (args.graph and headline) else "stream", "input_sets": n_sets},
        "kernels_ms": {k_: round(v, 4) for k_, v in ms.items()},
        "fwd_tokens_per_s": round(tokens / ((ms["select"] + ms["fwd"]) * 1e-3), 1),
        "roofline": roof(dominant),
        "roofline_fwd": roof("fwd"),
        "roofline_bwd": roof("bwd"),
        "roofline_all": {k_: roof(k_)["frac"] for k_ in ("fwd", "fwd_saving_for_bwd", "bwd_dq", "bwd_dkv", "bwd_dq_dkv", "bwd",
                                                          "bwd_gate", "select")},
        "traffic_source": (f"profiles/{w.name}_hbm_traffic.txt" if traffic else None),
    }
    if not args.shape:
        # the layer around the attention (output projection + residual + LayerNorm, every position): HBM-bound by design
        ms_op = R.timed(R.stage_fn("out_proj"), reps)
        sz, Dm = (4 if w.dtype == "fp32" else 2), w.H * w.d
        op_bytes = (3 * w.B * w.L * Dm + Dm * Dm) * sz
        out["out_proj_ln"] = {"ms": round(ms_op, 4), "bound": "hbm", "achieved": round(op_bytes / (ms_op * 1e-3) / 1e9, 1),
                              "peak": 8000.0, "unit": "GB/s", "frac": round(op_bytes / (ms_op * 1e-3) / 8e12, 4),
                              "traffic": traffic.get("out_proj"), "algorithmic_mb": round(op_bytes / 1e6, 1),
                              "tflops": round(2.0 * w.B * w.L * Dm * Dm / (ms_op * 1e-3) / 1e12, 1)}
    if ms_dense is not None:
        flops_dense = 4.0 * w.d * cnt["nnz_dense"]
        out["dense_causal"] = {"ms": round(ms_dense, 4), "tokens_per_s": round(tokens / (ms_dense * 1e-3), 1),
                               "tflops": round(flops_dense / (ms_dense * 1e-3) / 1e12, 2),
                               "sparse_fwd_speedup": round(ms_dense / (ms["select"] + ms["fwd"]), 3)}
    return out, R


def cpu_baseline(R):
    """The CPU oracle on a bounded sample of the same workload (reported, not a target)."""
    import oracle
    w, x = R.w, R.x
    threads = oracle.num_threads()
    total_pairs = w.B * w.H

    def run_oracle(n_pairs):
        prs = np.linspace(0, total_pairs - 1, n_pairs).astype(np.int32)
        t0 = time.perf_counter()
        sel_ref = oracle.select_blocks(x.Q, x.K, x.valid_len, w.block, w.topk, bh_list=prs)
        sel_ref = np.where(sel_ref == -2, -1, sel_ref)
        oracle.attn_fwd(x.Q, x.K, x.V, x.valid_len, sel_ref, x.gate_w, x.gate_b, w.block, w.topk, w.window,
                        bh_list=prs, stis_block=w.stis_block)
        oracle.attn_bwd(x.Q, x.K, x.V, x.valid_len, sel_ref, x.gate_w, x.gate_b, x.dO, w.block, w.topk,
                        w.window, bh_list=prs, stis_block=w.stis_block)
        dt_ = time.perf_counter() - t0
        toks = float(sum(int(x.valid_len[int(bh) // w.H]) for bh in prs)) / w.H
        return dt_, toks

    n_pairs = min(total_pairs, threads)
    cpu_s, sample_tokens = run_oracle(n_pairs)
    if cpu_s < 8.0 and n_pairs < total_pairs:  # aim at about 15 s of CPU work
        n_pairs = min(total_pairs, max(n_pairs + 1, int(n_pairs * 15.0 / max(cpu_s, 1e-3))))
        cpu_s, sample_tokens = run_oracle(n_pairs)
    cpu_model = "unknown"
    try:
        for line in open("/proc/cpuinfo"):
            if line.startswith("model name"):
                cpu_model = line.split(":", 1)[1].strip()
                break
    except OSError:
        pass
    return {"value": round(sample_tokens / cpu_s, 2), "unit": "tokens/s", "cores": threads, "cpu": cpu_model,
            "kind": "oracle",
            "sample": f"{n_pairs} of {total_pairs} (row, head) pairs, select+fwd+bwd, {cpu_s:.1f} s; "
                      f"tokens counted as pairs/H * valid_len"}


def run_positions(args, torch, B):
    """bench.py --stage positions: the path under the selection rule as the paper prints it (Sec. 3.4, Eq. 8-13
    per position, grouped key/value heads) at the paper's own setting (Appendix E: hidden 64 over 8 heads, 4
    key/value groups, compression blocks of 32 with stride 16, selection blocks of 16, k = 4, window 8, mask block
    1, fp32, lengths U[20,200], batch 2048): blossom_select_positions, blossom_attn_fwd_positions,
    blossom_attn_bwd_positions, each timed alone with HIP events, and the three as one training step."""
    dev = torch.device("cuda:0")
    Bn, H, G, L, d, l, s_, lsel, k, w = 2048, 8, 4, 200, 8, 32, 16, 16, 4, 8
    g = torch.Generator(device="cpu").manual_seed(2512)
    rnd = lambda *shape: torch.randn(shape, generator=g).to(dev)
    Q, dO = rnd(Bn, H, L, d), rnd(Bn, H, L, d)
    K, V = rnd(Bn, G, L, d), rnd(Bn, G, L, d)
    vl = torch.randint(20, L + 1, (Bn,), generator=g, dtype=torch.int32).to(dev)
    gw, gb = (0.02 * torch.randn((H, 2 * d), generator=g)).to(dev), torch.zeros(H, device=dev)
    p_sel = B.Params(Bn, H, L, d, lsel, k, 1, B.F32)
    p = B.Params(Bn, H, L, d, lsel, k, w, B.F32, stis_mode=1, stis_block=1)
    sel = B.select_positions(p_sel, G, l, s_, Q, K, vl)
    need = torch.empty(max(16, B.select_positions_workspace_bytes(p_sel, G, l, s_)), dtype=torch.uint8, device=dev)
    f = B.attn_fwd_positions(p, G, Q, K, V, vl, sel, gw, gb, want_branches=True)
    ws = torch.empty(max(16, B.workspace_bytes(p, B.WS_BWD)), dtype=torch.uint8, device=dev)
    bo = B.attn_bwd_positions(p, G, Q, K, V, vl, sel, gw, gb, f, dO, ws=ws)
    fns = {"select_positions": lambda: B.select_positions(p_sel, G, l, s_, Q, K, vl, sel_pos=sel, ws=need),
           "fwd_positions": lambda: B.attn_fwd_positions(p, G, Q, K, V, vl, sel, gw, gb, out=f),
           "bwd_positions": lambda: B.attn_bwd_positions(p, G, Q, K, V, vl, sel, gw, gb, f, dO, out=bo, ws=ws)}
    fns["step"] = lambda: [fn() for fn in (fns["select_positions"], fns["fwd_positions"], fns["bwd_positions"])]
    ms = {}
    for name, fn in fns.items():
        for _ in range(max(1, args.warmup)):
            fn()
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for _ in range(args.steps):
            fn()
        e1.record()
        torch.cuda.synchronize()
        ms[name] = round(e0.elapsed_time(e1) / args.steps, 4)
    tokens = int(vl.sum().item())
    sel_bytes = (Q.numel() + K.numel()) * 4 + sel.numel() * 4
    print(json.dumps({"stage": "positions", "shape": f"B={Bn} H={H} G={G} L={L} d={d} l={l} s={s_} l'={lsel} k={k} w={w} "
                                                      f"mask block 1 fp32, lens U[20,{L}]",
                      "ms": ms, "tokens_per_step": tokens, "step_tokens_per_s": round(tokens / (ms["step"] * 1e-3), 1),
                      "select_positions_gbs": round(sel_bytes / (ms["select_positions"] * 1e-3) / 1e9, 1)}))


def run_ceiling(args, torch, B):
    """bench.py --stage ceiling: the stripped tile loop of the matrix-core forward (blossom_probe), one
    launch per kind, timed with HIP events; prints what each pipe alone and all of them together cost per
    64-query x 64-key tile and what that means for the cfg4 forward (311296 such tiles on 256 CUs)."""
    dev = torch.device("cuda:0")
    n = B.probe_bytes(0) // 2
    g = torch.Generator(device=dev).manual_seed(7)
    K = (torch.randn(n, device=dev, generator=g) / 8).to(torch.bfloat16)
    V = (torch.randn(n, device=dev, generator=g) / 8).to(torch.bfloat16)
    sink = torch.empty(B.probe_bytes(1) // 4, dtype=torch.float32, device=dev)
    iters = 500
    # a launch: PROBE_WORKGROUPS workgroups x 2 wavefronts x iters steps of 32 keys x 64 queries
    #         = PROBE_WORKGROUPS x iters tiles of 64 x 64; 256 CUs work on them in parallel
    tiles_per_cu = B.PROBE_WORKGROUPS * iters / 256.0
    cfg4_tiles_per_cu = 311296 / 256.0      # 16384 query blocks x 19 tiles (3 window + 16 selected)
    flops_alg = 284.4e9                     # cfg4 forward, algorithmic (4 d pairs)
    res = {}
    for kind, name in enumerate(PROBE_KINDS):
        B.probe(kind, K, V, sink, iters)
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for _ in range(3):
            B.probe(kind, K, V, sink, iters)
        e1.record()
        torch.cuda.synchronize()
        ns_tile = e0.elapsed_time(e1) / 3 * 1e6 / tiles_per_cu
        us_fwd = ns_tile * cfg4_tiles_per_cu * 1e-3
        res[name] = {"cu_ns_per_64x64_tile": round(ns_tile, 1), "cfg4_fwd_us_at_this_rate": round(us_fwd, 1),
                     "cfg4_fwd_mfma_roofline_frac_at_this_rate": round(flops_alg / (us_fwd * 1e-6) / 2.5e15, 3)}
    mf = res[PROBE_KINDS[0]]["cu_ns_per_64x64_tile"]
    # kind 0 issues 18 matrix instructions of 32x32x16 per wavefront step, 36 per tile and CU over 4 SIMDs
    res["mfma_sustained_tflops"] = round(36 * 32 * 32 * 16 * 2 / (mf * 1e-9) * 256 / 1e12, 1)
    res["staging_bytes_per_clk_per_cu_at_2p1GHz"] = round(16384 / res[PROBE_KINDS[5]]["cu_ns_per_64x64_tile"] / 2.1, 1)
    print(json.dumps({"stage": "ceiling", "iters": iters, "probe": res}))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--workload", default="cfg4", help="cfg1..cfg5 (shapes of the five parity configs)")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--no-second-workload", action="store_true",
                    help="skip the L=1024 training-step workload (cfg5) that the default run times next to cfg4")
    ap.add_argument("--input-sets", type=int, default=3,
                    help="independent seeded input sets the timed steps rotate over, so that a small workload is not "
                         "served from the 256 MB last-level cache (one set with --stage and --graph)")
    ap.add_argument("--graph", action="store_true",
                    help="capture the step (select + forward + backward) in a HIP graph once and time its replays")
    ap.add_argument("--shape", default="",
                    help="overrides of the workload's fields, e.g. B=32,H=8,L=2000,len_lo=2000,len_hi=2000 "
                         "(the efficiency-study shapes of the paper's Appendix B); the JSON line names them")
    ap.add_argument("--stis-block", type=int, default=0,
                    help="0: short-term mask = causal window (default); N >= 1: all of Eq. 15 with mask block N")
    ap.add_argument("--no-dense", action="store_true")
    ap.add_argument("--stage", choices=STAGES + ["ceiling", "positions"], default=None,
                    help="profiling aid: run only this stage --steps times (after the others ran once) "
                         "and print its average time; the headline line is not produced.  'ceiling' runs the "
                         "stripped tile loop of the matrix-core forward (what each pipe costs alone and together)")
    args = ap.parse_args()
    if args.gpus != 1:
        print("bench.py: this build runs on ONE GPU; --gpus N with N > 1 is not supported "
              "(every (row, head) pair is independent in selection, forward and backward: rows shard over GPUs "
              "with no exchange in forward and one small all-reduce of the gate gradients in backward).",
              file=sys.stderr)
        sys.exit(2)

    import torch
    from paper_2512_13368_amd import binding as B
    from paper_2512_13368_amd.inputs import WORKLOADS, bf16_bits, make_inputs, with_shape

    torch.cuda.set_device(torch.device("cuda:0"))
    if args.stage == "ceiling":
        run_ceiling(args, torch, B)
        return
    if args.stage == "positions":
        run_positions(args, torch, B)
        return
    w = WORKLOADS[args.workload]
    if args.stis_block:
        w = with_shape(w, stis_block=args.stis_block)
    if args.shape:
        kv = dict(t.split("=") for t in args.shape.split(","))
        w = with_shape(w, name=w.name + "*", **{k_: int(v_) for k_, v_ in kv.items()})
    mods = (torch, B, make_inputs, bf16_bits)
    n_sets = 1 if (args.stage or args.graph) else max(1, args.input_sets)

    if args.stage:
        R = Runner(w, 1, *mods)
        R.step()  # every buffer a later stage reads is filled once
        fn = R.stage_fn(args.stage)
        for _ in range(args.warmup):
            fn()
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for _ in range(args.steps):
            fn()
        e1.record()
        torch.cuda.synchronize()
        print(json.dumps({"stage": args.stage, "workload": w.name, "steps": args.steps,
                          "avg_ms": round(e0.elapsed_time(e1) / args.steps, 4)}))
        return

    res, R = measure_workload(w, args, mods, n_sets, headline=True)
    out = {
        "metric": "sparse-attn fwd+bwd tokens/sec (select + forward + backward per step)",
        "value": res.pop("tokens_per_s"),
        "unit": "tokens/s",
        "n_gpus": 1,
        "steps": args.steps,
        "warmup": args.warmup,
        "ms_per_step": res.pop("ms_per_step"),
        "higher_is_better": True,
        "scaling": "weak",
        "vs_baseline": None,
        "dtype": w.dtype if w.dtype == "bf16" else "f32",
        "data": "synthetic",
    }
    out.update(res)
    # ---- CPU oracle on a bounded sample of the same workload ----
    if not args.no_cpu_baseline:
        out["cpu_baseline"] = cpu_baseline(R)
    # ---- the metric's other half: the L=1024 training step (cfg5), timed the same way in the same run ----
    if args.workload == "cfg4" and not (args.shape or args.stis_block or args.no_second_workload or args.graph):
        del R
        torch.cuda.empty_cache()
        res5, R5 = measure_workload(WORKLOADS["cfg5"], args, mods, n_sets, headline=False)
        out["l1024_training_step"] = res5
        # ---- and the paper's own regime: the short-sequence recommender shape (cfg2: L = 200, fp32), same step ----
        del R5
        torch.cuda.empty_cache()
        res2, _ = measure_workload(WORKLOADS["cfg2"], args, mods, n_sets, headline=False)
        out["l200_training_step"] = res2
    print(json.dumps(out))


if __name__ == "__main__":
    main()
