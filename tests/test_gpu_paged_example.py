"""The serving example: histories taken in as prompts and grown item by item give what one prompt over everything gives."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("users,history,steps", [(5, 70, 3), (1, 300, 2), (40, 33, 40)])
def test_serving_example(users, history, steps):
    spec = importlib.util.spec_from_file_location("serve_paged", os.path.join(ROOT, "examples", "serve_paged.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    # both sides are within the bf16 bound (2e-2 of values up to about 3) of the exact result
    assert module.main(users, history, steps) <= 0.12


@pytest.mark.gpu
@pytest.mark.parametrize("users,history", [(5, 70), (3, 700), (12, 33)])
def test_a_steps_branches_against_64_bits(users, history, monkeypatch):
    """Full attention and the blend of the two branches of one new item, from what the cache holds, at the operators' usual bound."""
    import torch

    spec = importlib.util.spec_from_file_location("serve_paged", os.path.join(ROOT, "examples", "serve_paged.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    H, G, d, page, topk, window = module.HEADS, module.GROUPS, module.DIM, module.PAGE, module.TOPK, module.WINDOW
    lengths = [max(1, history * (u + 1) // users) for u in range(users)]
    g = torch.Generator(device="cuda").manual_seed(7)
    items = lambda n: torch.randn(n, module.WIDTH, generator=g, device="cuda").bfloat16()
    layer = module.Layer(users, history + 1)
    layer.prompt(items(sum(lengths)), lengths)
    seen = {}
    append, select = layer.append, layer.select
    monkeypatch.setattr(layer, "append", lambda *a: seen.setdefault("q", append(*a)))
    monkeypatch.setattr(layer, "select", lambda *a: seen.setdefault("listed", select(*a)))
    full, blossom = layer.step(items(users))
    q, (table, listed) = seen["q"].double().cpu(), seen["listed"]
    table, listed = table.cpu().tolist(), listed.tolist()
    K, V, pages, gate = layer.K_cache.double().cpu(), layer.V_cache.double().cpu(), layer.table.tolist(), layer.gate_w.double().cpu()

    def attend(x, ids, n, grp, first=0):
        at = [(ids[j // page], j % page) for j in range(first, n)]
        k, v = (torch.stack([c[i, grp, r] for i, r in at]) for c in (K, V))
        return torch.softmax(k @ x * d**-0.5, 0) @ v

    want_full, want = torch.zeros(users, H, d, dtype=torch.float64), torch.zeros(users, H, d, dtype=torch.float64)
    for u in range(users):
        n = lengths[u] + 1
        newest = (n - 1) // page
        for grp in range(G):
            heads = range(grp * (H // G), (grp + 1) * (H // G))
            # the newest page, and of the earlier ones those whose mean keys score best, in their order
            score = {i: float(K[pages[u][i], grp].mean(0) @ q[u, list(heads)].sum(0)) for i in range(newest)}
            mine = table[u][grp][:min(topk, newest + 1)]
            places = [pages[u].index(i) for i in mine]
            assert places == sorted(places) and places[-1] == newest and len(set(places)) == len(places) == min(topk, newest + 1)
            left = [x for i, x in score.items() if i not in places]
            assert not left or max(left) <= min(score[i] for i in places[:-1]) + 1e-3
            assert listed[u] == (len(places) - 1) * page + (n - 1) % page + 1
            for h in heads:
                want_full[u, h] = attend(q[u, h], pages[u], n, grp)
                lt, st = attend(q[u, h], mine, listed[u], grp), attend(q[u, h], pages[u], n, grp, max(0, n - window))
                alpha = torch.sigmoid((torch.cat([lt, st]) * gate[h]).sum())
                want[u, h] = alpha * lt + (1 - alpha) * st
    for got, ref in ((full, want_full), (blossom, want)):
        off = (got.double().cpu() - ref).abs() - 2e-2 * (ref.abs() + ref.pow(2).mean().sqrt())
        assert float(off.max()) <= 0, f"off by {float(off.max()):.3g} beyond the bound"
