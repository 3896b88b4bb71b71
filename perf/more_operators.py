"""Timed cases of continuing a history in several ways at once: trees of drafted tokens, and beams, over a paged key/value cache.

  append   kv_append_tree: drafted tokens go to the cache, each rotated by its place in the tree (its depth), not by its slot
  tree     attn_tree: each drafted token attends the cached history and the drafted tokens that its mask names, its ancestors
  accept   kv_accept: of a drafted tree, the tokens that were kept move down to follow the history
  fork     kv_fork and kv_copy_pages: sequences go on from the beams that were chosen; full pages are shared, partly filled ones copied
  beam     beam_select: the best continuations over a history's beams and the whole vocabulary (the items)

Each has a plain form here in elementary torch operations, and the framework's own calls where `own` is set.  Shapes are those of
the repository's workloads (`inputs.WORKLOADS`: heads, head sizes, lengths, blocks as pages) and generic ones with grouped heads.
"""
import math

import torch

own = False


def _paged(name, op, seqs, heads, groups, dim, page, dtype, new, past, window=0, keep=0):
    """new, past: (least, most) drafted tokens of a sequence, and positions that its cache holds before; window: a token sees the
    cached positions that lie less than that far behind it (0: all); keep: at most that many drafted tokens are accepted."""
    c = {"op": op, "S": seqs, "H": heads, "G": groups, "d": dim, "page": page, "dtype": dtype, "new_lo": new[0], "new_hi": new[1],
         "past_lo": past[0], "past_hi": past[1], "window": window, "keep": keep}
    return dict(c, name=name) if name else c


def _fork(name, histories, beams, groups, dim, page, dtype, past, made, grow):
    """past: (least, most) positions of a history, shared by its beams; made: (least, most) positions that beams have made since."""
    c = {"op": "fork", "B": histories, "W": beams, "G": groups, "d": dim, "page": page, "dtype": dtype, "past_lo": past[0],
         "past_hi": past[1], "made_lo": made[0], "made_hi": made[1], "grow": grow}
    return dict(c, name=name) if name else c


def _beam(name, histories, beams, best, vocab, dtype, pad, ends):
    """pad: a row of logits begins at every multiple of that many elements; ends: of 100 beams, how many are at their end."""
    c = {"op": "beam", "B": histories, "W": beams, "K": best, "V": vocab, "dtype": dtype, "pad": pad, "ends": ends}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a few drafts for a handful of short histories: launches and the host path (workload cfg1's heads and lengths)
        _paged("tree_tiny_fp32", "tree", 4, 2, 2, 32, 8, "fp32", (3, 6), (9, 49)),
        # a serving batch, 16 drafts each (workload cfg3's heads and lengths)
        _paged("tree_batch_bf16", "tree", 64, 4, 4, 64, 32, "bf16", (16, 16), (99, 1007)),
        # drafts for one user's very long history, alone on the card
        _paged("tree_one_bf16", "tree", 1, 32, 8, 128, 64, "bf16", (26, 26), (131040, 131040)),
        # full trees over 16 long sequences with grouped heads
        _paged("tree_wide_bf16", "tree", 16, 32, 8, 128, 16, "bf16", (33, 64), (4000, 8100)),
        # drafted tokens on their way into the cache between two layers' attention: a handful, and a batch of full trees
        _paged("append_tiny_fp32", "append", 4, 2, 2, 32, 8, "fp32", (3, 6), (9, 49)),
        _paged("append_trees_bf16", "append", 128, 32, 8, 128, 16, "bf16", (33, 64), (100, 2000)),
        # the accepted path of each tree, a layer's caches: short drafts, and full trees of many sequences
        _paged("accept_tiny_fp32", "accept", 4, 2, 2, 32, 8, "fp32", (3, 6), (9, 49), keep=4),
        _paged("accept_trees_bf16", "accept", 128, 32, 8, 128, 16, "bf16", (33, 64), (100, 2000), keep=12),
        # one history's four beams, and eight beams for each of 64 histories (workload cfg3's heads, longer histories)
        _fork("fork_tiny_fp32", 1, 4, 2, 32, 8, "fp32", (9, 49), (1, 9), 1),
        _fork("fork_batch_bf16", 64, 8, 4, 64, 32, "bf16", (99, 4000), (1, 40), 1),
        # one history's four beams over a small catalogue
        _beam("beam_tiny_fp32", 1, 4, 4, 1682, "fp32", 1, 0),
        # eight beams for each of 64 histories over a large one, rows as a product padded to 64 columns leaves them
        _beam("beam_large_bf16", 64, 8, 16, 152063, "bf16", 64, 5),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "append", "accept", "fork", "beam", "beam"])
    groups, share = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
    dim = rng.choice([8, 16, 32, 64, 64, 128, 128])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    size = 4 if dtype == "fp32" else 2
    if op == "beam":
        vocab = _log(rng, 20, 400_000)
        beams, best = _log(rng, 1, 32), _log(rng, 1, 32)
        # no more bytes than the largest listed case reads
        histories = _log(rng, 1, max(1, min(256, 150_000_000 // (vocab * beams * size))))
        return _beam(None, histories, beams, best, vocab, dtype, rng.choice([1, 1, 8, 64]), rng.choice([0, 10, 50]))
    if op == "fork":
        past, made = _log(rng, 1, 8192), _log(rng, 1, 64)
        beams = _log(rng, 2, 32)
        cells = 300_000_000 // (groups * dim * 2 * size)  # positions that the caches hold
        histories = _log(rng, 1, max(1, min(128, cells // (past + beams * (made + 2 * page)))))
        return _fork(None, histories, beams, groups, dim, page, dtype, (past // rng.choice([1, 2, 10]), past), (made // 2, made),
                     rng.choice([1, 1, 4, 17]))
    new = _log(rng, 1, 64)
    new_lo = max(1, new // rng.choice([1, 1, 2, 8]))
    past = _log(rng, 1, 131072 if op == "tree" else 4096)
    past_lo = past // rng.choice([1, 2, 10])
    if op != "tree":
        cells = 400_000_000 // (groups * dim * 2 * size)
        seqs = _log(rng, 1, max(1, min(256, cells // (past + new))))
        return _paged(None, op, seqs, groups * share, groups, dim, page, dtype, (new_lo, new), (past_lo, past), keep=min(new, rng.choice([1, 4, 16])))
    # no more bytes than a listed case reads, and no more products (an eighth of them where these run in 32 bits)
    by_bytes = 450_000_000 // ((past + new) * groups * dim * 2 * size)
    while share > 1 and new * groups * share * (past + new) * dim > (8_000_000_000 if dtype == "bf16" else 1_000_000_000):
        share //= 2
    by_pairs = (16_000_000_000 if dtype == "bf16" else 2_000_000_000) // (new * groups * share * (past + new) * dim)
    seqs = _log(rng, 1, max(1, min(256, by_bytes, by_pairs)))
    return _paged(None, op, seqs, groups * share, groups, dim, page, dtype, (new_lo, new), (past_lo, past),
                  rng.choice([0, 0, 0, _log(rng, 1, past + new)]))


def _spread(lo, hi, n):
    """n whole numbers evenly spread between two bounds."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


class _State:
    pass


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def prepare(case, seed):
    s, dev = _State(), torch.device("cuda:0")
    s.case = case
    g = torch.Generator(device=dev).manual_seed(seed)
    order = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(_dtype(case))

    {"beam": _prepare_beam, "fork": _prepare_fork}.get(case["op"], _prepare_tree)(s, case, dev, g, order, normal)
    return s


def _prepare_tree(s, case, dev, g, order, normal):
    S, H, G, d, page, op = (case[k] for k in ("S", "H", "G", "d", "page", "op"))
    mixed = torch.randperm(S, generator=order)
    new = torch.tensor(_spread(case["new_lo"], case["new_hi"], S))[mixed]
    past = torch.tensor(_spread(case["past_lo"], case["past_hi"], S))[mixed.flip(0)]
    T = int(new.sum())
    s.new_max = int(new.max())
    width = (case["new_hi"] + case["past_hi"] + page - 1) // page
    n_pages = S * width + 3
    # the pages of a sequence lie anywhere in the cache
    s.page_table = torch.randperm(n_pages, generator=g, device=dev)[:S * width].view(S, width).to(torch.int32)
    s.K_cache, s.V_cache = normal(n_pages, G, page, d), normal(n_pages, G, page, d)
    s.kv_len = (past + new).to(torch.int32).to(dev)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
    s.cu_seqlens = cu.to(torch.int32).to(dev)
    # a drafted token goes on from the history (parent -1) or from an earlier drafted one, mostly a recent one
    N = s.new_max
    back = (torch.rand(S, N, generator=order) ** 2 * (torch.arange(N) + 1)).long() + 1
    parent = (torch.arange(N) - back).clamp(min=-1)
    seen = torch.eye(N, dtype=torch.bool).repeat(S, 1, 1)  # [S, token, its ancestors and itself]
    for i in range(1, N):
        up = parent[:, i]
        seen[:, i] |= seen[torch.arange(S), up.clamp(min=0)] & (up >= 0)[:, None]
    masks = (seen.long() << torch.arange(N)).sum(-1)
    row = torch.arange(T)
    seq = torch.searchsorted(cu, row, right=True) - 1
    s.tree_mask = masks[seq, row - cu[seq]].to(dev)
    cap = width * page
    if op == "append":
        qkv = normal(T, (H + 2 * G) * d)  # as one projection of the drafted tokens leaves them
        s.Q, s.K, s.V = (x.unflatten(1, (-1, d)) for x in qkv.split([H * d, G * d, G * d], 1))
        angle = torch.arange(cap, device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, device=dev, dtype=torch.float64) / d)
        s.rope_cos, s.rope_sin = angle.cos().float(), angle.sin().float()
        s.Q_rot = torch.empty(T, H, d, dtype=_dtype(case), device=dev)
    elif op == "tree":
        s.Q = normal(T, H, d)
        s.O = torch.empty(T, H, d, dtype=_dtype(case), device=dev)
        s.lse = torch.empty(T, H, dtype=torch.float32, device=dev)
    else:
        # a path down each tree: ascending drafted tokens, as many as were kept, then -1
        kept = (torch.rand(S, generator=order) * (torch.minimum(new, torch.tensor(case["keep"])) + 1)).long()
        lots = torch.rand(S, N, generator=order)
        lots = torch.where(torch.arange(N) < new[:, None], lots, torch.full_like(lots, 2.0))
        among = lots.argsort(1).argsort(1) < kept[:, None]
        path = torch.where(among, torch.arange(N), N).sort(1).values[:, :case["keep"]]
        s.keep = torch.where(path < N, path, -1).to(torch.int32).to(dev)
        s.new_len = torch.empty(S, dtype=torch.int32, device=dev)
    if own:  # the parameters and the workspace that a program keeps between calls
        from paper_2512_13368_amd import binding as B
        s.p = B.PagedParams(S=S, T=T, H=H, G=G, d=d, page=page, n_pages=n_pages, max_pages=width, dtype=B.F32 if case["dtype"] == "fp32" else B.BF16,
                            window=case["window"])
        if op == "tree":
            s.ws = torch.empty(max(16, B.paged_workspace_bytes(s.p, B.WS_TREE)), dtype=torch.uint8, device=dev)


def _prepare_fork(s, case, dev, g, order, normal):
    B_, W, G, d, page, grow = (case[k] for k in ("B", "W", "G", "d", "page", "grow"))
    N = B_ * W
    past = torch.tensor(_spread(case["past_lo"], case["past_hi"], B_))[torch.randperm(B_, generator=order)]
    made = torch.tensor(_spread(case["made_lo"], case["made_hi"], B_))[torch.randperm(B_, generator=order)]
    length = (past + made).repeat_interleave(W)
    # a history's full pages are held by all of its beams; what comes after is each one's own
    full = (past // page).repeat_interleave(W)
    held = (length + page - 1) // page
    width = (case["past_hi"] + case["made_hi"] + grow + page - 1) // page + 1
    i = torch.arange(width)
    first = (torch.arange(N) // W) * W
    ranks = torch.where(i < full[:, None], first[:, None] * width + i, torch.arange(N)[:, None] * width + i)
    ranks = torch.where(i < held[:, None], ranks, -1)
    used = torch.unique(ranks[ranks >= 0])
    n_pages = int((past // page).sum() + W * (made // page + 2).sum()) + 2 * N + N * (grow // page) + 3  # some are nobody's
    place = torch.randperm(n_pages, generator=order)[:used.numel()]
    ids = torch.full((N * width + 1,), -1, dtype=torch.int64)
    ids[used] = place
    table = ids[ranks]
    s.page_table = table.to(torch.int32).to(dev)
    s.kv_len = length.to(torch.int32).to(dev)
    s.refs = torch.bincount(table[table >= 0], minlength=n_pages).to(torch.int32).to(dev)
    # the chosen beams: good ones are gone on from several times, others never
    good = (torch.rand(B_, W, generator=order) ** 2 * W).long()
    s.parent = (good + torch.arange(B_)[:, None] * W).view(-1).to(torch.int32).to(dev)
    s.K_cache, s.V_cache = normal(n_pages, G, page, d), normal(n_pages, G, page, d)
    s.new_table = torch.empty_like(s.page_table)
    s.new_len = torch.empty_like(s.kv_len)
    s.new_refs = torch.empty_like(s.refs)
    s.copies = torch.empty(N, 3, dtype=torch.int32, device=dev)
    s.missing = torch.empty(1, dtype=torch.int32, device=dev)
    if own:
        from paper_2512_13368_amd import binding as B
        s.p = B.PagedParams(S=N, T=N, H=G, G=G, d=d, page=page, n_pages=n_pages, max_pages=width, dtype=B.F32 if case["dtype"] == "fp32" else B.BF16)
        s.ws = torch.empty(max(16, B.fork_workspace_bytes(s.p, N)), dtype=torch.uint8, device=dev)


def _prepare_beam(s, case, dev, g, order, normal):
    B_, W, K, V = (case[k] for k in ("B", "W", "K", "V"))
    stride = -(-V // case["pad"]) * case["pad"]
    rows = torch.empty(B_ * W, stride, dtype=_dtype(case), device=dev)
    rows.normal_(0.0, 2.5, generator=g)
    # items that a history holds already are ruled out
    out = torch.randint(0, V, (B_ * W, max(1, V // 50)), generator=g, device=dev)
    rows.scatter_(1, out, -math.inf)
    s.logits = rows[:, :V]
    s.score = -torch.rand(B_, W, generator=g, device=dev) * 12.0
    s.eos = V - 1 if case["ends"] else -1
    s.ended = torch.rand(B_, W, generator=g, device=dev) * 100.0 < case["ends"] if case["ends"] else None
    s.parent = torch.empty(B_, K, dtype=torch.int32, device=dev)
    s.token = torch.empty(B_, K, dtype=torch.int32, device=dev)
    s.out_score = torch.empty(B_, K, dtype=torch.float32, device=dev)
    s.out_ended = torch.empty(B_, K, dtype=torch.bool, device=dev)
    if own:
        from paper_2512_13368_amd import binding as B
        s.p = B.BeamParams(B=B_, W=W, K=K, V=V, dtype=B.F32 if case["dtype"] == "fp32" else B.BF16, eos=s.eos)
        s.ws = torch.empty(max(16, B.beam_workspace_bytes(s.p)), dtype=torch.uint8, device=dev)


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "tree": _plain_tree, "accept": _plain_accept, "fork": _plain_fork, "beam": _plain_beam}[s.case["op"]](s)


def _own(s):
    from paper_2512_13368_amd import binding as B
    op = s.case["op"]
    if op == "append":
        B.kv_append_tree(s.p, s.K, s.V, s.K_cache, s.V_cache, s.page_table, s.cu_seqlens, s.kv_len, s.tree_mask, Q=s.Q,
                         rope=(s.rope_cos, s.rope_sin), Q_rot=s.Q_rot)
        return {"K_cache": s.K_cache, "V_cache": s.V_cache, "Q_rot": s.Q_rot}
    if op == "tree":
        B.attn_tree(s.p, s.Q, s.K_cache, s.V_cache, s.page_table, s.cu_seqlens, s.kv_len, s.tree_mask, O=s.O, lse=s.lse, ws=s.ws)
        return {"O": s.O, "lse": s.lse}
    if op == "accept":
        B.kv_accept(s.p, s.keep, s.K_cache, s.V_cache, s.page_table, s.cu_seqlens, s.kv_len, new_len=s.new_len)
        return {"K_cache": s.K_cache, "V_cache": s.V_cache, "new_len": s.new_len}
    if op == "fork":
        B.kv_fork(s.p, s.parent, s.page_table, s.kv_len, s.refs, grow=s.case["grow"], new_table=s.new_table, new_len=s.new_len,
                  new_refs=s.new_refs, copies=s.copies, missing=s.missing, ws=s.ws)
        B.kv_copy_pages(s.p, s.copies, s.K_cache, s.V_cache)
        return {"table": s.new_table, "len": s.new_len, "refs": s.new_refs, "copies": s.copies, "missing": s.missing,
                "K_cache": s.K_cache, "V_cache": s.V_cache}
    B.beam_select(s.p, s.logits, s.score, ended=s.ended, parent=s.parent, token=s.token, out_score=s.out_score, out_ended=s.out_ended, ws=s.ws)
    return {"parent": s.parent, "token": s.token, "score": s.out_score, "ended": s.out_ended}


def _tokens(s):
    """Of each drafted token: its sequence, its place among that one's drafted tokens, how many those are, and which of them it sees."""
    cu = s.cu_seqlens.long()
    t = torch.arange(s.tree_mask.shape[0], device=cu.device)
    seq = (t[:, None] >= cu[None, 1:]).sum(1)
    at, count = t - cu[seq], (cu[1:] - cu[:-1])[seq]
    i = torch.arange(64, device=cu.device)
    bits = ((s.tree_mask[:, None] >> i) & 1).bool() & (i < count[:, None])
    others = (bits & (i != at[:, None])).sum(1)  # so many positions behind the history it stands
    return seq, at, count, bits, others


def _rotate(x, c, s):
    x = x.float()
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack([x0 * c - x1 * s, x0 * s + x1 * c], -1).flatten(-2)


def _plain_append(s):
    page, dt = s.case["page"], s.Q.dtype
    seq, at, count, _, others = _tokens(s)
    past = s.kv_len.long()[seq] - count
    slot, pos = past + at, past + others
    where, row = s.page_table.long()[seq, slot // page], slot % page
    c, sn = s.rope_cos[pos][:, None], s.rope_sin[pos][:, None]
    s.K_cache[where, :, row] = _rotate(s.K, c, sn).to(dt)
    s.V_cache[where, :, row] = s.V
    return {"K_cache": s.K_cache, "V_cache": s.V_cache, "Q_rot": _rotate(s.Q, c, sn).to(dt)}


def _plain_tree(s):
    case = s.case
    S, H, G, d, w = (case[k] for k in ("S", "H", "G", "d", "window"))
    R, N = H // G, s.new_max
    table = s.page_table.long()
    K, V = (c[table].permute(0, 2, 1, 3, 4).flatten(2, 3).float() for c in (s.K_cache, s.V_cache))  # [S, G, positions, d]
    seq, at, count, bits, others = _tokens(s)
    # a padded batch of the packed rows
    q = torch.zeros(S, N, H, d, device=K.device)
    q[seq, at] = s.Q.float()
    q = q.view(S, N, G, R, d).permute(0, 2, 3, 1, 4).reshape(S, G, R * N, d)
    logits = torch.matmul(q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(S, G, R, N, -1)
    past = (s.kv_len.long()[seq] - count)[:, None]
    j = torch.arange(K.shape[2], device=K.device)
    sees = j < past
    if w:
        sees = sees & (j > past + others[:, None] - w)
    drafted = torch.gather(bits, 1, (j - past).clamp(0, 63)) & (j >= past) & (j - past < 64)
    seen = torch.zeros(S, N, K.shape[2], dtype=torch.bool, device=K.device)
    seen[seq, at] = sees | drafted
    logits.masked_fill_(~seen[:, None, None], -math.inf)
    m = logits.amax(-1, keepdim=True).clamp_(min=-3e38)
    e = logits.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    O = torch.matmul(e, V[:, :, None]) / total.clamp(min=1e-38)
    O = O.permute(0, 3, 1, 2, 4)[seq, at].reshape(-1, H, d)
    lse = (m + total.log()).squeeze(-1).permute(0, 3, 1, 2)[seq, at].reshape(-1, H)
    return {"O": O.to(s.Q.dtype), "lse": lse}


def _plain_accept(s):
    page, keep = s.case["page"], s.keep.long()
    count = (s.cu_seqlens[1:] - s.cu_seqlens[:-1]).long()
    before = torch.cat([torch.full_like(keep[:, :1], -1), keep[:, :-1]], 1)
    kept = ((keep > before) & (keep < count[:, None])).long().cumprod(1).bool()  # ascending, up to the first that is not
    past = s.kv_len.long() - count
    b, i = kept.nonzero(as_tuple=True)
    src, to = past[b] + keep[b, i], past[b] + i
    src_page, to_page = s.page_table.long()[b, src // page], s.page_table.long()[b, to // page]
    # (indexing copies: every row is read before one is written)
    s.K_cache[to_page, :, to % page] = s.K_cache[src_page, :, src % page]
    s.V_cache[to_page, :, to % page] = s.V_cache[src_page, :, src % page]
    s.new_len.copy_(past + kept.sum(1))
    return {"K_cache": s.K_cache, "V_cache": s.V_cache, "new_len": s.new_len}


def _plain_fork(s):
    page, grow = s.case["page"], s.case["grow"]
    table, refs, n_pages = s.page_table.long(), s.refs.long(), s.refs.numel()
    S, width = table.shape
    cap = width * page
    parent = s.parent.long()
    alive = (parent >= 0) & (parent < S)
    q = parent.clamp(0, S - 1)
    N = parent.numel()
    me = torch.arange(N, device=table.device)
    length = torch.where(alive, s.kv_len.long()[q].clamp(0, cap), 0)
    full, part = length // page, length % page
    need = torch.where(alive, ((length + grow).clamp(max=cap) + page - 1) // page, 0)
    first = torch.full((S,), N, dtype=torch.int64, device=table.device).scatter_reduce_(0, q, torch.where(alive, me, N), "amin")
    i = torch.arange(width, device=table.device)
    old = table[q]
    there = (old >= 0) & (old < n_pages)
    shared = (i < full[:, None]) & there
    mine = (i >= full[:, None]) & (i < need[:, None])
    kept = mine & there & (first[q] == me)[:, None] & (refs[old.clamp(0, n_pages - 1)] == 1)
    fresh = mine & ~kept
    new = torch.where(shared | kept, old, -1)

    def holders(t):
        ok = (t >= 0) & (t < n_pages)
        return torch.zeros(n_pages, dtype=torch.int64, device=t.device).scatter_add_(0, t.clamp(0, n_pages - 1).view(-1), ok.long().view(-1))

    refs = refs - holders(table) + holders(new)
    # pages that nobody holds and that no copy reads are given out, the lowest first, to the sequences in order
    at_full = full.clamp(max=width - 1)[:, None]
    copied = (part > 0) & torch.gather(fresh & there, 1, at_full)[:, 0] & (full < width)
    source = torch.where(copied, torch.gather(old, 1, at_full)[:, 0], -1)
    free = (refs == 0) & (holders(source) == 0)
    ids = torch.argsort((~free).to(torch.int8), stable=True)
    nth = fresh.view(-1).long().cumsum(0).view(N, width) - 1
    n_free, asked = free.sum(), fresh.sum()
    given = torch.where(fresh & (nth < n_free), ids[nth.clamp(0, n_pages - 1)], -1)
    new = torch.where(fresh, given, new)
    refs = refs + holders(given)
    target = torch.gather(new, 1, at_full)[:, 0]
    copied = copied & (target >= 0)
    none = torch.full_like(part, -1)
    copies = torch.stack([torch.where(copied, source, none), torch.where(copied, target, none), torch.where(copied, part, 0)], 1)
    # the copies themselves: rows that are not copied stay as they are
    rows = (torch.arange(page, device=table.device) < copies[:, 2:])[copied][:, None, :, None]
    src, dst = source[copied], target[copied]
    s.K_cache[dst] = torch.where(rows, s.K_cache[src], s.K_cache[dst])
    s.V_cache[dst] = torch.where(rows, s.V_cache[src], s.V_cache[dst])
    return {"table": new.int(), "len": length.int(), "refs": refs.int(), "copies": copies.int(),
            "missing": (asked - n_free).clamp(min=0).int().view(1), "K_cache": s.K_cache, "V_cache": s.V_cache}


def _plain_beam(s):
    B_, W, K, V = (s.case[k] for k in ("B", "W", "K", "V"))
    x = s.logits.float() + 0.0  # (-0 is 0)
    x = torch.where(x.isnan(), -math.inf, x)
    m = x.amax(1, keepdim=True)
    lse = m.double() + (x - m).double().exp().sum(1, keepdim=True).log()  # in 64 bits: two beams' scores may be near each other
    # the best of each row: logits in order, equal ones by their item
    bits = x.view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (V - 1 - torch.arange(V, device=x.device))
    k = min(K, V)
    token = V - 1 - (key.topk(k, dim=1).values & 0xFFFFFFFF)
    score = s.score.double().view(-1, 1) + (torch.gather(x, 1, token).double() - lse)
    if s.ended is not None:  # a beam at its end goes on as it is, in one way
        ended = s.ended.view(-1, 1)
        only = torch.where(torch.arange(k, device=x.device) == 0, s.score.double().view(-1, 1), -math.inf)
        score, token = torch.where(ended, only, score), torch.where(ended, s.eos, token)
    score = torch.where(score.isnan(), -math.inf, score).view(B_, W * k)
    if W * k < K:
        score = torch.cat([score, torch.full((B_, K - W * k), -math.inf, dtype=score.dtype, device=x.device)], 1)
    score, at = score.sort(dim=1, descending=True, stable=True)
    score, at = score[:, :K], at[:, :K]
    none = score == -math.inf
    parent = at // k + torch.arange(B_, device=x.device)[:, None] * W
    token = torch.gather(token.view(B_, W * k), 1, at.clamp(max=W * k - 1))
    over = token == s.eos
    if s.ended is not None:
        over = over | s.ended.view(-1)[parent.clamp(max=B_ * W - 1)]
    return {"parent": torch.where(none, -1, parent).int(), "token": torch.where(none, -1, token).int(), "score": score.float(), "ended": over & ~none}


def _counts(case):
    n = case["S"]
    return _spread(case["new_lo"], case["new_hi"], n), _spread(case["past_lo"], case["past_hi"], n)[::-1]


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    op = case["op"]
    if op == "beam":
        rows = case["B"] * case["W"] * (100 - case["ends"]) / 100
        # a difference, an exponential, a sum and a comparison for each logit
        return {"bytes": rows * case["V"] * size + case["B"] * (case["W"] * 4 + case["K"] * 13), "flops": 4 * rows * case["V"]}
    G, d, page = case["G"], case["d"], case["page"]
    if op == "fork":
        N = case["B"] * case["W"]
        entries = N * ((case["past_lo"] + case["past_hi"] + case["made_lo"] + case["made_hi"]) // 2 // page + 1)
        # old and new tables; half the beams go on from another's page, half of which is filled
        return {"bytes": 8 * entries + 24 * N + N // 2 * 4 * (page // 2) * G * d * size, "flops": entries}
    S, H = case["S"], case["H"]
    new, past = _counts(case)
    T = sum(new)
    if op == "append":
        return {"bytes": 2 * T * (H + 2 * G) * d * size + T * (d * 4 + 8), "flops": 3 * T * (H + G) * d}
    if op == "accept":
        # half of what may be kept is, on the average, K and V read and written
        return {"bytes": sum(min(n, case["keep"]) for n in new) // 2 * 4 * G * d * size + S * 8, "flops": 0}
    w = case["window"]
    pairs = sum(n * (min(b, w) if w else b) + n * (n + 1) // 4 for n, b in zip(new, past))
    keys = sum((min(b, w) if w else b) + n for n, b in zip(new, past))
    return {"bytes": 2 * keys * G * d * size + 2 * T * H * d * size + T * H * 4 + 8 * T, "flops": 4 * d * H * pairs}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "tree": _exact_tree, "accept": _exact_accept, "fork": _exact_fork, "beam": _exact_beam}[case["op"]](s, case)


def _trees(s):
    """(sequence, first token, tokens, history) of each, on the host."""
    cu, n = s.cu_seqlens.tolist(), s.kv_len.tolist()
    return [(b, cu[b], cu[b + 1] - cu[b], n[b] - (cu[b + 1] - cu[b])) for b in range(len(n))]


def _lineage(s, lo, n):
    """bool [n, n]: does the token see the other?"""
    masks = s.tree_mask[lo:lo + n].tolist()
    return torch.tensor([[m >> i & 1 == 1 for i in range(n)] for m in masks], device=s.tree_mask.device)


def _exact_append(s, case):
    page = case["page"]
    K, V = s.K_cache.double(), s.V_cache.double()
    Q = torch.empty(s.Q.shape, dtype=torch.float64, device=K.device)
    for b, lo, n, past in _trees(s):
        at = past + _lineage(s, lo, n).fill_diagonal_(False).sum(1)
        turn = torch.complex(s.rope_cos[at].double(), s.rope_sin[at].double())[:, None]  # a pair of channels as one number
        slot = torch.arange(past, past + n, device=K.device)
        to = s.page_table[b].long()[slot // page]

        def turned(x):
            z = torch.view_as_complex(x[lo:lo + n].double().contiguous().unflatten(-1, (-1, 2)))
            return torch.view_as_real(z * turn).flatten(-2)

        Q[lo:lo + n] = turned(s.Q)
        K[to, :, slot % page] = turned(s.K)
        V[to, :, slot % page] = s.V[lo:lo + n].double()
    return {"K_cache": K, "V_cache": V, "Q_rot": Q}


def _exact_tree(s, case):
    H, G, d, page, w = (case[k] for k in ("H", "G", "d", "page", "window"))
    dev = s.Q.device
    O = torch.zeros(s.Q.shape, dtype=torch.float64, device=dev)
    lse = torch.empty(s.Q.shape[:2], dtype=torch.float64, device=dev)
    for b, lo, n, past in _trees(s):
        sees = _lineage(s, lo, n)
        depth = sees.clone().fill_diagonal_(False).sum(1)
        j = torch.arange(past + n, device=dev)
        back = (past + depth)[:, None] - j[:past]
        history = back < w if w else torch.ones_like(back, dtype=torch.bool)
        hidden = ~torch.cat([history, sees], 1)
        ids = s.page_table[b].long()[j // page]
        for g in range(G):
            k, v = s.K_cache[ids, g, j % page].double(), s.V_cache[ids, g, j % page].double()
            for h in range(g * (H // G), (g + 1) * (H // G)):
                x = (s.Q[lo:lo + n, h].double() @ k.t()) / d ** 0.5
                x.masked_fill_(hidden, float("-inf"))
                lse[lo:lo + n, h] = torch.logsumexp(x, 1)
                O[lo:lo + n, h] = torch.exp(x - lse[lo:lo + n, h, None]) @ v
    return {"O": O, "lse": lse}


def _exact_accept(s, case):
    page = case["page"]
    K, V = s.K_cache.double(), s.V_cache.double()
    table, keep = s.page_table.tolist(), s.keep.tolist()
    lens, src, dst = [], [], []
    for b, _, n, past in _trees(s):
        m = 0
        while m < len(keep[b]) and keep[b][m] >= 0:
            src.append((table[b][(past + keep[b][m]) // page], (past + keep[b][m]) % page))
            dst.append((table[b][(past + m) // page], (past + m) % page))
            m += 1
        lens.append(past + m)
    if src:
        a, b = (torch.tensor(x, device=K.device).t() for x in (src, dst))
        K[b[0], :, b[1]], V[b[0], :, b[1]] = s.K_cache[a[0], :, a[1]].double(), s.V_cache[a[0], :, a[1]].double()
    return {"K_cache": K, "V_cache": V, "new_len": torch.tensor(lens, dtype=torch.int32, device=K.device)}


def _exact_fork(s, case):
    page, grow = case["page"], case["grow"]
    table, lens, refs, parent = (x.tolist() for x in (s.page_table, s.kv_len, s.refs, s.parent))
    width = len(table[0])
    before = list(refs)
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] -= 1
    went, rows, copies, wanted = set(), [], [], []
    for n, q in enumerate(parent):
        full, part = divmod(lens[q], page)
        need = -(-min(lens[q] + grow, width * page) // page)
        row = table[q][:full] + [-1] * (width - full)
        eldest = q not in went
        went.add(q)
        copies.append([-1, -1, 0])
        for i in range(full, need):
            p = table[q][i]
            if eldest and p >= 0 and before[p] == 1:
                row[i] = p
                continue
            wanted.append((n, i))
            if i == full and part and p >= 0:
                copies[n] = [p, -1, part]
        for p in row:
            if p >= 0:
                refs[p] += 1
        rows.append(row)
    sources = {c[0] for c in copies}
    spare = iter([p for p, r in enumerate(refs) if r == 0 and p not in sources])
    missing = 0
    for n, i in wanted:
        p = next(spare, -1)
        rows[n][i] = p
        missing += p < 0
        if p >= 0:
            refs[p] += 1
        if copies[n][2] and i == lens[parent[n]] // page:
            copies[n] = [copies[n][0], p, copies[n][2]] if p >= 0 else [-1, -1, 0]
    K, V = s.K_cache.double(), s.V_cache.double()
    for a, b, k in copies:
        if b >= 0:
            K[b, :, :k], V[b, :, :k] = s.K_cache[a, :, :k].double(), s.V_cache[a, :, :k].double()

    def whole(x):
        return torch.tensor(x, dtype=torch.int32, device=K.device)

    return {"table": whole(rows), "len": whole([lens[q] for q in parent]), "refs": whole(refs), "copies": whole(copies),
            "missing": whole([missing]), "K_cache": K, "V_cache": V}


def _exact_beam(s, case):
    B_, W, K, V = (case[k] for k in ("B", "W", "K", "V"))
    parent = torch.full((B_, K), -1, dtype=torch.int32, device=s.score.device)
    token, score = parent.clone(), torch.full((B_, K), float("-inf"), dtype=torch.float64, device=s.score.device)
    ended = torch.zeros(B_, K, dtype=torch.bool, device=s.score.device)
    for b in range(B_):
        p = torch.log_softmax(s.logits[b * W:(b + 1) * W].double(), 1) + s.score[b].double()[:, None]
        if s.ended is not None:
            alone = torch.full_like(p, float("-inf"))
            alone[:, s.eos] = s.score[b].double()
            p = torch.where(s.ended[b][:, None], alone, p)
        v, i = p.flatten().sort(descending=True, stable=True)
        v, i = v[:K], i[:K]
        i = i[v > float("-inf")]
        k = i.numel()
        parent[b, :k], token[b, :k], score[b, :k] = (i // V + b * W).int(), (i % V).int(), v[:k]
        ended[b, :k] = i % V == s.eos
    return {"parent": parent, "token": token, "score": score, "ended": ended}
