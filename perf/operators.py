"""Timed cases of serving from a paged key/value cache: what a program that answers online calls per request.

Histories live in pages of a cache between requests.  Three operators work on it:
  append  kv_append: the keys and values of new tokens go to their places in the cache, keys and queries rotated by position
  prompt  attn_prompt: causal attention of each sequence's new tokens over its cached keys, their own among them
  decode  attn_decode: the same for one new token a sequence

Each has a plain form here in elementary torch operations in 32 bits, and the framework's own call where `own` is set.
Shapes are those of the repository's workloads (`inputs.WORKLOADS`: heads, head sizes, lengths, blocks as pages, top-k) and
generic ones with grouped heads; lengths are ragged, and queries, keys and values come as slices of one fused projection.
"""
import math

import torch

own = False


def _case(name, op, seqs, heads, groups, dim, page, dtype, new, past, window=0, topk=0):
    """new, past: (least, most) tokens that a sequence adds, and that its cache holds before; window: a query sees that many
    positions up to its own (0: all); topk: decode attends that many pages, chosen per key/value head (0: all)."""
    c = {"op": op, "S": seqs, "H": heads, "G": groups, "d": dim, "page": page, "dtype": dtype, "new_lo": new[0], "new_hi": new[1],
         "past_lo": past[0], "past_hi": past[1], "window": window, "topk": topk}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a handful of short histories get one item each: launches and the host path (workload cfg1's heads and lengths)
        _case("append_tiny_fp32", "append", 4, 2, 2, 32, 8, "fp32", (1, 1), (9, 49)),
        # one token for each of 128 sequences, between two layers' attention
        _case("append_step_bf16", "append", 128, 32, 8, 128, 16, "bf16", (1, 1), (100, 4095)),
        # the prompts of 16 new sequences of every length up to 2047
        _case("append_prompt_bf16", "append", 16, 32, 8, 128, 16, "bf16", (1, 2047), (0, 0)),
        # the next item of a few short histories
        _case("decode_tiny_fp32", "decode", 4, 2, 2, 32, 8, "fp32", (1, 1), (9, 49)),
        # a serving batch of ragged histories, a key head to each query head (workload cfg3's heads and lengths)
        _case("decode_batch_bf16", "decode", 128, 4, 4, 64, 32, "bf16", (1, 1), (99, 1023)),
        # the long-term branch for one new item: 16 chosen pages of a history of 8192 for each head (workload cfg4)
        _case("decode_selected_bf16", "decode", 16, 8, 8, 64, 64, "bf16", (1, 1), (8128, 8191), topk=16),
        # 16 long sequences with grouped heads
        _case("decode_long_bf16", "decode", 16, 32, 8, 128, 16, "bf16", (1, 1), (4000, 8190)),
        # one user's very long history, alone on the card
        _case("decode_one_bf16", "decode", 1, 32, 8, 128, 64, "bf16", (1, 1), (131070, 131070)),
        # a batch of short histories scored anew (workload cfg2's heads and lengths)
        _case("prompt_short_fp32", "prompt", 256, 2, 2, 32, 16, "fp32", (20, 200), (0, 0)),
        # ragged prompts packed together, some of them a few tokens
        _case("prompt_ragged_bf16", "prompt", 32, 16, 4, 64, 32, "bf16", (7, 1997), (0, 0)),
        # a chunk of 512 tokens over a cached past, sliding window
        _case("prompt_chunk_bf16", "prompt", 4, 32, 8, 128, 16, "bf16", (512, 512), (1000, 16000), window=4096),
        # long prompts in one piece
        _case("prompt_long_bf16", "prompt", 2, 32, 8, 128, 64, "bf16", (6001, 8191), (0, 0)),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prompt", "prompt"])
    groups, share = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8])
    dim = rng.choice([8, 16, 32, 64, 64, 128, 128])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    heads = groups * share
    size = 4 if dtype == "fp32" else 2
    if op == "append":
        seqs = _log(rng, 1, 256)
        if rng.random() < 0.5:
            hi = past = _log(rng, 1, 4096)
            return _case(None, op, seqs, heads, groups, dim, page, dtype, (1, 1), (max(0, past // rng.choice([1, 8])), hi))
        hi = _log(rng, 2, max(2, min(4096, 32768 // seqs)))
        return _case(None, op, seqs, heads, groups, dim, page, dtype, (1, hi), (0, rng.choice([0, hi])))
    if op == "decode":
        past = _log(rng, 1, 131072)
        # no more bytes than the largest listed case reads
        seqs = _log(rng, 1, max(1, min(256, 500_000_000 // (past * groups * dim * 2 * size))))
        kind = rng.choice(["all", "all", "window", "pages"])
        topk = min(rng.randint(2, 16), past // page + 1) if kind == "pages" else 0
        return _case(None, op, seqs, heads, groups, dim, page, dtype, (1, 1), (past // rng.choice([1, 2, 10]), past),
                     _log(rng, 1, past + 1) if kind == "window" else 0, topk)
    hi = _log(rng, 2, 8192)
    past = rng.choice([0, 0, hi, 3 * hi])
    # pairs of the padded square, over all heads: an eighth of the largest listed one where products run in 32 bits
    pairs = (400_000_000 if dtype == "fp32" else 3_000_000_000) // (heads * hi * (hi + past))
    seqs = _log(rng, 1, max(1, min(256, pairs)))
    while heads > groups and heads * hi * (hi + past) > 4_000_000_000:
        heads //= 2
        heads -= heads % groups
    return _case(None, op, seqs, max(heads, groups), groups, dim, page, dtype, (max(1, hi // rng.choice([1, 3, 100])), hi), (past // 2, past),
                 rng.choice([0, 0, _log(rng, 1, hi + past)]))


def _lengths(case):
    """(new, past) of each sequence, in an order that prepare() mixes: evenly spread between the case's bounds."""
    n = case["S"]

    def spread(lo, hi):
        return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]

    return spread(case["new_lo"], case["new_hi"]), spread(case["past_lo"], case["past_hi"])


class _State:
    pass


def prepare(case, seed):
    s, dev = _State(), torch.device("cuda:0")
    S, H, G, d, page, op = (case[k] for k in ("S", "H", "G", "d", "page", "op"))
    s.case = case
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    g = torch.Generator(device=dev).manual_seed(seed)
    order = torch.Generator().manual_seed(seed)
    new, past = _lengths(case)
    mixed = torch.randperm(S, generator=order)
    new, past = torch.tensor(new)[mixed], torch.tensor(past)[mixed]
    total = new + past
    T = int(new.sum())
    s.new_max = int(new.max())

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(dt)

    # the pages of a sequence lie anywhere in the cache; some are nobody's
    width = (case["new_hi"] + case["past_hi"] + page - 1) // page
    n_pages = S * width + 3
    pages = torch.randperm(n_pages, generator=g, device=dev)[:S * width].view(S, width).to(torch.int32)
    s.max_pages = width
    s.K_cache, s.V_cache = normal(n_pages, G, page, d), normal(n_pages, G, page, d)
    if case["topk"]:
        # each key/value head lists its own pages in ascending order, the newest among them
        last = (total - 1) // page
        at = torch.arange(width)
        lots = torch.rand(S, G, width, generator=order)
        lots = torch.where(at < last[:, None, None], lots, torch.full_like(lots, -1.0))
        lots = torch.where(at == last[:, None, None], torch.full_like(lots, 2.0), lots)
        k = s.max_pages = min(case["topk"], width)
        chosen = lots.topk(k, dim=2).indices
        real = torch.minimum(last + 1, torch.tensor(k))[:, None, None]  # pages that there are: the others come last
        chosen = torch.where(torch.arange(k) < real, chosen, torch.full_like(chosen, width)).sort(dim=2).values
        ids = torch.cat([pages, torch.full((S, 1), -1, dtype=torch.int32, device=dev)], 1)
        pages = ids[torch.arange(S, device=dev)[:, None, None], chosen.to(dev)].contiguous()
        total = (real[:, 0, 0] - 1) * page + (total - 1) % page + 1
    s.page_table = pages
    s.kv_len = total.to(torch.int32).to(dev)
    s.cu_seqlens = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).to(torch.int32).to(dev)

    if op == "append":
        # Q, K and V as one projection of the new tokens leaves them
        qkv = normal(T, (H + 2 * G) * d)
        s.Q, s.K, s.V = (x.unflatten(1, (-1, d)) for x in qkv.split([H * d, G * d, G * d], 1))
        pos = torch.arange(width * page, device=dev, dtype=torch.float64)
        angle = pos[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, device=dev, dtype=torch.float64) / d)
        s.rope_cos, s.rope_sin = angle.cos().float(), angle.sin().float()
        s.Q_rot = torch.empty(T, H, d, dtype=dt, device=dev)
    else:
        s.Q = normal(T, H, d)
        s.O = torch.empty(T, H, d, dtype=dt, device=dev)
        s.lse = torch.empty(T, H, dtype=torch.float32, device=dev)
    if own:  # the parameters and the workspace that a program keeps between calls
        from paper_2512_13368_amd import binding as B
        s.p = B.PagedParams(S=S, T=T, H=H, G=G, d=d, page=page, n_pages=n_pages, max_pages=s.max_pages,
                            dtype=B.F32 if dt == torch.float32 else B.BF16, window=case["window"], table_per_head=int(case["topk"] > 0))
        if op != "append":
            which = B.WS_DECODE if op == "decode" else B.WS_PROMPT
            s.ws = torch.empty(max(16, B.paged_workspace_bytes(s.p, which)), dtype=torch.uint8, device=dev)
    return s


def run(s):
    op = s.case["op"]
    if own:
        from paper_2512_13368_amd import binding as B
        if op == "append":
            B.kv_append(s.p, s.K, s.V, s.K_cache, s.V_cache, s.page_table, s.cu_seqlens, s.kv_len, Q=s.Q, rope=(s.rope_cos, s.rope_sin),
                        Q_rot=s.Q_rot)
            return {"K_cache": s.K_cache, "V_cache": s.V_cache, "Q_rot": s.Q_rot}
        if op == "decode":
            B.attn_decode(s.p, s.Q, s.K_cache, s.V_cache, s.page_table, s.kv_len, O=s.O, lse=s.lse, ws=s.ws)
        else:
            B.attn_prompt(s.p, s.Q, s.K_cache, s.V_cache, s.page_table, s.cu_seqlens, s.kv_len, O=s.O, lse=s.lse, ws=s.ws)
        return {"O": s.O, "lse": s.lse}
    return {"append": _plain_append, "decode": _plain_decode, "prompt": _plain_prompt}[op](s)


def _rotate(x, c, s):
    x = x.float()
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack([x0 * c - x1 * s, x0 * s + x1 * c], -1).flatten(-2)


def _plain_append(s):
    page, dt = s.case["page"], s.Q.dtype
    cu, kv_len = s.cu_seqlens.long(), s.kv_len.long()
    t = torch.arange(s.Q.shape[0], device=s.Q.device)
    seq = (t[:, None] >= cu[None, 1:]).sum(1)
    pos = kv_len[seq] - cu[seq + 1] + t
    where, slot = s.page_table.long()[seq, pos // page], pos % page
    c, sn = s.rope_cos[pos][:, None], s.rope_sin[pos][:, None]
    s.K_cache[where, :, slot] = _rotate(s.K, c, sn).to(dt)
    s.V_cache[where, :, slot] = s.V
    return {"K_cache": s.K_cache, "V_cache": s.V_cache, "Q_rot": _rotate(s.Q, c, sn).to(dt)}


def _gathered(s, cache):
    """[S, G, positions, d] in 32 bits: the listed pages one after another."""
    table = s.page_table.long().clamp(min=0)
    if table.dim() == 2:
        return cache[table].permute(0, 2, 1, 3, 4).flatten(2, 3).float()
    groups = torch.arange(table.shape[1], device=table.device)
    return cache[table, groups[None, :, None]].flatten(2, 3).float()


def _softmax_product(logits, seen, V):
    """(O, lse) of logits where `seen`; a row that sees nothing gives 0 and -inf."""
    logits = logits.masked_fill_(~seen, -math.inf)
    m = logits.amax(-1, keepdim=True).clamp_(min=-3e38)
    e = logits.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, V) / total.clamp(min=1e-38), (m + total.log()).squeeze(-1)


def _plain_decode(s):
    case = s.case
    S, H, G, d = (case[k] for k in ("S", "H", "G", "d"))
    K, V = _gathered(s, s.K_cache), _gathered(s, s.V_cache)
    q = s.Q.float().view(S, G, H // G, d)
    logits = torch.matmul(q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    j = torch.arange(K.shape[2], device=K.device)
    n = s.kv_len.long()[:, None]
    seen = j < n
    if case["window"]:
        seen = seen & (j >= n - case["window"])
    O, lse = _softmax_product(logits, seen[:, None, None], V)
    return {"O": O.reshape(S, H, d).to(s.Q.dtype), "lse": lse.reshape(S, H)}


def _plain_prompt(s):
    case = s.case
    S, H, G, d = (case[k] for k in ("S", "H", "G", "d"))
    R, N, T = H // G, s.new_max, s.Q.shape[0]
    K, V = _gathered(s, s.K_cache), _gathered(s, s.V_cache)
    cu, kv_len = s.cu_seqlens.long(), s.kv_len.long()
    i = torch.arange(N, device=K.device)
    row = (cu[:-1, None] + i).clamp(max=T - 1)  # [S, N]: the token of each place of a padded batch
    q = s.Q.float()[row].view(S, N, G, R, d).permute(0, 2, 3, 1, 4).reshape(S, G, R * N, d)
    logits = torch.matmul(q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(S, G, R, N, -1)
    pos = (kv_len - (cu[1:] - cu[:-1]))[:, None] + i
    j = torch.arange(K.shape[2], device=K.device)
    seen = j <= pos[..., None]
    if case["window"]:
        seen = seen & (j > pos[..., None] - case["window"])
    O, lse = _softmax_product(logits, seen[:, None, None], V[:, :, None])
    # back to packed rows
    t = torch.arange(T, device=K.device)
    seq = (t[:, None] >= cu[None, 1:]).sum(1)
    at = t - cu[seq]
    O = O.permute(0, 3, 1, 2, 4)[seq, at].reshape(T, H, d)
    return {"O": O.to(s.Q.dtype), "lse": lse.permute(0, 3, 1, 2)[seq, at].reshape(T, H)}


def _visible(case):
    """(query, key) pairs of one head over all sequences, and the keys that any query sees."""
    pairs = keys = 0
    w = case["window"]
    new, past = _lengths(case)
    if case["op"] == "decode":
        for b, a in zip(past, new):
            n = a + b
            if case["topk"]:
                n = min(n, (min(case["topk"], (n - 1) // case["page"] + 1) - 1) * case["page"] + (n - 1) % case["page"] + 1)
            n = min(n, w) if w else n
            pairs, keys = pairs + n, keys + n
        return pairs, keys
    for b, a in zip(past, new):
        if not w:
            pairs, keys = pairs + a * b + a * (a + 1) // 2, keys + a + b
        else:
            rising = max(0, min(a, w - b))  # queries that see all there is
            pairs += rising * b + rising * (rising + 1) // 2 + (a - rising) * w
            keys += min(a + b, a + w - 1)
    return pairs, keys


def work(case):
    S, H, G, d = (case[k] for k in ("S", "H", "G", "d"))
    size = 4 if case["dtype"] == "fp32" else 2
    T = sum(_lengths(case)[0])
    if case["op"] == "append":
        # Q, K, V read, Q_rot and both caches' rows written; a row of each table a token
        return {"bytes": 2 * T * (H + 2 * G) * d * size + T * d * 4, "flops": 3 * T * (H + G) * d}
    pairs, keys = _visible(case)
    return {"bytes": 2 * keys * G * d * size + 2 * T * H * d * size + T * H * 4, "flops": 4 * d * H * pairs}


def exact(case, seed):
    s = prepare(case, seed)
    H, G, d, page, w = (case[k] for k in ("H", "G", "d", "page", "window"))
    cu, kv_len = s.cu_seqlens.tolist(), s.kv_len.tolist()
    if case["op"] == "append":
        K_cache, V_cache = s.K_cache.double(), s.V_cache.double()
        Q_rot = torch.empty(s.Q.shape, dtype=torch.float64, device=s.Q.device)
        for b in range(case["S"]):
            lo, hi = cu[b], cu[b + 1]
            at = torch.arange(kv_len[b] - (hi - lo), kv_len[b], device=s.Q.device)
            turn = torch.complex(s.rope_cos[at].double(), s.rope_sin[at].double())[:, None]  # a pair of channels as one number
            to = s.page_table[b].long()[at // page]
            for src, dst in ((s.Q, None), (s.K, K_cache)):
                z = torch.view_as_complex(src[lo:hi].double().contiguous().unflatten(-1, (-1, 2)))
                z = torch.view_as_real(z * turn).flatten(-2)
                if dst is None:
                    Q_rot[lo:hi] = z
                else:
                    dst[to, :, at % page] = z
            V_cache[to, :, at % page] = s.V[lo:hi].double()
        return {"K_cache": K_cache, "V_cache": V_cache, "Q_rot": Q_rot}
    O = torch.zeros(s.Q.shape, dtype=torch.float64, device=s.Q.device)
    lse = torch.empty(s.Q.shape[:2], dtype=torch.float64, device=s.Q.device)
    for b in range(case["S"]):
        lo, hi = (b, b + 1) if case["op"] == "decode" else (cu[b], cu[b + 1])
        n = kv_len[b]
        j = torch.arange(n, device=s.Q.device)
        back = torch.arange(n - (hi - lo), n, device=s.Q.device)[:, None] - j  # how far a key lies behind a query
        hidden = (back < 0) | (back >= w) if w else back < 0
        for g in range(G):
            table = s.page_table[b, g] if s.page_table.dim() == 3 else s.page_table[b]
            ids = table.long()[j // page]
            k, v = s.K_cache[ids, g, j % page].double(), s.V_cache[ids, g, j % page].double()
            for h in range(g * (H // G), (g + 1) * (H // G)):
                x = (s.Q[lo:hi, h].double() @ k.t()) / d ** 0.5
                x.masked_fill_(hidden, float("-inf"))
                lse[lo:hi, h] = torch.logsumexp(x, 1)
                O[lo:hi, h] = torch.exp(x - lse[lo:hi, h, None]) @ v
    return {"O": O, "lse": lse}
