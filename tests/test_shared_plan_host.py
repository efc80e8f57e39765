"""The planner of attention over shared prefixes, without a device: every query token meets each of its keys exactly once, items
are what the kernel can take, and partial results do not overlap."""
import random

import pytest
import torch

import paper_2511_07423_b200 as syn
from workloads.configs import ModelShape

STAGE = 128


def shape(hd, hq, hkv):
    return ModelShape("plan", 1, 128, hq, hkv, hd, 128, 1000)


def tree_batch(rng, ctx_own, chunk, levels, scattered=True):
    """levels: [(pages, group)]: every `group` neighbours share `pages` more; then own pages.  Returns tables, ctx lens, pages."""
    n = len(ctx_own)
    rows = [[] for _ in range(n)]
    at = 0
    for pages, group in levels:
        for g in range(0, n, group):
            ids = list(range(at, at + pages))
            at += pages
            for i in range(g, min(n, g + group)):
                rows[i] += ids
    ctx = [16 * len(r) + c for r, c in zip(rows, ctx_own)]
    for i in range(n):
        need = -(-(ctx[i] + chunk[i]) // 16) - len(rows[i])
        rows[i] += list(range(at, at + need))
        at += need
    perm = list(range(at))
    if scattered:
        rng.shuffle(perm)
    most = max(map(len, rows))
    table = torch.tensor([[perm[x] for x in r] + [-7] * (most - len(r)) for r in rows], dtype=torch.int32)
    off = torch.tensor([0] + chunk).cumsum(0).to(torch.int32)
    return table, torch.tensor(ctx, dtype=torch.int32), off, at


CASES = [   # own cached tokens, chunks, levels of (pages, group), (hd, hq, hkv), SMs
    ([5, 0, 40], [1, 1, 1], [(20, 3)], (128, 32, 8), 148),
    ([0] * 9, [32] * 9, [(8, 9)], (64, 16, 2), 148),
    ([100, 7, 300, 17, 90, 1], [3, 9, 1, 32, 2, 8], [(64, 6), (9, 2)], (128, 40, 8), 148),
    ([1] * 40, [7] * 40, [(30, 40), (12, 5), (8, 1)], (128, 6, 2), 16),
    ([10, 20], [4, 4], [(7, 2)], (128, 8, 1), 148),                    # too little in common for a node
    ([2000], [17], [(0, 1)], (64, 32, 8), 148),
    ([5] * 33, [1, 2, 3] * 11, [(100, 33), (40, 11)], (128, 7, 1), 5),
    ([70, 3, 0, 9], [2, 30, 1, 7], [(25, 4), (9, 2)], (64, 6, 2), 1),     # one CTA has it all
    ([9] * 64, [1] * 64, [(90, 64)], (128, 8, 8), 148),                # one query head to a kv head
]


@pytest.mark.parametrize("case", CASES)
def test_every_token_meets_its_keys_once(case):
    own, chunk, levels, (hd, hq, hkv), n_sm = case
    rng = random.Random(len(own))
    table, ctx, off, n_pages = tree_batch(rng, own, chunk, levels)
    T, G = int(off[-1]), hq // hkv
    p = syn.plan_shared_host(shape(hd, hq, hkv), n_pages, torch.zeros(T, dtype=torch.int32), off, table, ctx, n_sm=n_sm)
    items = [dict(zip(("q_tok", "n_tok", "kvh", "req", "kv_begin", "kv_end", "q_pos0", "base", "mode"), r)) for r in p["items"].tolist()]
    assert p["n_cta"] <= n_sm and p["cta_begin"].tolist()[0] == 0 and p["cta_begin"].tolist()[-1] == len(items)
    assert all(a < b for a, b in zip(p["cta_begin"].tolist(), p["cta_begin"].tolist()[1:]))
    req_of = [i for i in range(len(own)) for _ in range(chunk[i])]
    pos_of = [int(ctx[i]) + j for i in range(len(own)) for j in range(chunk[i])]
    met = {}          # (token, kv head) -> physical key slots, with multiplicity
    rows = {}         # row -> (token, kv head) of its first query head
    used = set()
    tile = 128 // G
    for it in items:
        tiles = 2 if it["mode"] == 2 else 1
        assert 1 <= it["n_tok"] <= tile * tiles and it["mode"] in (0, 1, 2, 3) and (tiles == 1 or it["n_tok"] > tile)
        assert it["kv_begin"] % 16 == 0 and it["kv_begin"] < it["kv_end"]
        stages = -(-(it["kv_end"] - it["kv_begin"]) // STAGE)
        copies = 2 if it["mode"] == 3 else 1
        assert copies == 1 or stages > 1
        span = range(it["base"], it["base"] + copies * it["n_tok"] * G)
        assert not used & set(span)
        used |= set(span)
        for j in range(it["n_tok"]):
            t = it["q_tok"] + j
            last = it["kv_end"] - 1 if it["q_pos0"] < 0 else min(it["kv_end"] - 1, it["q_pos0"] + j)
            assert it["q_pos0"] < 0 or it["q_pos0"] + j == pos_of[t]
            keys = range(it["kv_begin"], last + 1)
            met.setdefault((t, it["kvh"]), []).extend(int(table[it["req"], k // 16]) * 16 + k % 16 for k in keys)
            for c in range(copies):
                rows[it["base"] + (c * it["n_tok"] + j) * G] = (t, it["kvh"])
    want_parts = sorted((t, h, r) for r, (t, h) in rows.items())
    assert sorted(map(tuple, p["parts"].tolist())) == want_parts
    for t in range(T):
        r = req_of[t]
        want = sorted(int(table[r, k // 16]) * 16 + k % 16 for k in range(pos_of[t] + 1))
        for h in range(hkv):
            assert sorted(met[t, h]) == want
    shared_rows = {it["q_pos0"] for it in items}
    assert (-1 in shared_rows) == any(pages * 16 >= STAGE and group > 1 for pages, group in levels if len(own) > 1)


def test_shared_keys_count_once():
    table, ctx, off, n_pages = tree_batch(random.Random(1), [16] * 10, [1] * 10, [(100, 10)])
    p = syn.plan_shared_host(shape(128, 32, 8), n_pages, torch.zeros(10, dtype=torch.int32), off, table, ctx)
    assert p["taken"]
    assert p["stats"].kv_read_bytes == (1600 + 10 * 17) * 2 * 8 * 128 * 2
    plain = syn.plan_host(shape(128, 32, 8), n_pages, torch.zeros(10, dtype=torch.int32), off, table, ctx)["stats"]
    assert plain.kv_read_bytes == 10 * 1617 * 2 * 8 * 128 * 2
    assert p["stats"].kernel_launches == plain.kernel_launches + 1


def test_pages_that_are_not_full_or_not_cached_are_not_shared():
    # two requests on the same ten pages of which the second has cached 130 tokens: 8 full pages in common
    table = torch.tensor([[*range(12)], [*range(8), 20, 21, 22, 23]], dtype=torch.int32)
    ctx = torch.tensor([170, 130], dtype=torch.int32)
    off = torch.tensor([0, 1, 2], dtype=torch.int32)
    p = syn.plan_shared_host(shape(128, 32, 8), 30, torch.zeros(2, dtype=torch.int32), off, table, ctx)
    shared = [r for r in p["items"].tolist() if r[6] < 0]
    assert shared and {(r[4], r[5]) for r in shared} == {(0, 128)}
    ctx = torch.tensor([170, 127], dtype=torch.int32)       # the eighth page is not full
    p = syn.plan_shared_host(shape(128, 32, 8), 30, torch.zeros(2, dtype=torch.int32), off, table, ctx)
    assert not any(r[6] < 0 for r in p["items"].tolist()) and not p["taken"]


def test_nothing_shared_is_planned_as_ever():
    table, ctx, off, n_pages = tree_batch(random.Random(2), [500] * 4, [2] * 4, [])
    p = syn.plan_shared_host(shape(128, 32, 8), n_pages, torch.zeros(8, dtype=torch.int32), off, table, ctx)
    assert not p["taken"]
    try:
        syn.debug_set_attention(4)
        assert syn.plan_shared_host(shape(128, 32, 8), n_pages, torch.zeros(8, dtype=torch.int32), off, table, ctx)["taken"]
        syn.debug_set_attention(2)
        table, ctx, off, n_pages = tree_batch(random.Random(2), [5] * 40, [2] * 40, [(200, 40)])
        assert not syn.plan_shared_host(shape(128, 32, 8), n_pages, torch.zeros(80, dtype=torch.int32), off, table, ctx)["taken"]
    finally:
        syn.debug_set_attention(0)
    assert syn.plan_shared_host(shape(128, 32, 8), n_pages, torch.zeros(80, dtype=torch.int32), off, table, ctx)["taken"]


def test_a_few_long_requests_are_cut_finer():
    for own, heads in (([4149], (128, 14, 2)), ([10460], (128, 8, 1)), ([29589, 12000], (128, 14, 2))):
        table, ctx, off, n_pages = tree_batch(random.Random(5), own, [8] * len(own), [])
        p = syn.plan_shared_host(shape(*heads), n_pages, torch.zeros(8 * len(own), dtype=torch.int32), off, table, ctx)
        assert p["taken"] and not any(r[6] < 0 for r in p["items"].tolist())
        plain = syn.plan_host(shape(*heads), n_pages, torch.zeros(8 * len(own), dtype=torch.int32), off, table, ctx)["stats"]
        assert p["stats"].kv_read_bytes == plain.kv_read_bytes


def test_many_requests_in_a_chain_of_prefixes():
    # request i shares i * 8 pages with request i + 1: a path of nested runs
    n, rows = 60, []
    for i in range(n):
        rows.append(list(range(8 * min(i + 1, n))))
    most = 8 * n + 4
    at = 8 * n
    table = torch.full((n, most), 0, dtype=torch.int32)
    ctx = []
    for i, r in enumerate(rows):
        r = r + [at + i]
        table[i, :len(r)] = torch.tensor(r, dtype=torch.int32)
        ctx.append(16 * (len(r) - 1) + 3)
    off = torch.arange(n + 1, dtype=torch.int32)
    p = syn.plan_shared_host(shape(64, 8, 2), at + n, torch.zeros(n, dtype=torch.int32), off, table, torch.tensor(ctx, dtype=torch.int32))
    keys = {}
    for q_tok, n_tok, h, req, b, e, q0, base, mode in p["items"].tolist():
        for t in range(q_tok, q_tok + n_tok):
            if h == 0:
                keys[t] = keys.get(t, 0) + (e - b if q0 < 0 else min(e, ctx[t] + 1) - b)
    assert keys == {t: ctx[t] + 1 for t in range(n)}


@pytest.mark.parametrize("ctx,chunk,code", [([5], 33, -2), ([-1], 1, -1), ([160], 1, -5)])
def test_refusals_are_the_planners(ctx, chunk, code):
    with pytest.raises(syn.SynError) as e:
        syn.plan_shared_host(shape(128, 32, 8), 10, torch.zeros(chunk, dtype=torch.int32), torch.tensor([0, chunk], dtype=torch.int32),
                             torch.arange(10, dtype=torch.int32)[None], torch.tensor(ctx, dtype=torch.int32))
    assert e.value.code == code
    with pytest.raises(syn.SynError):
        syn.plan_shared_host(shape(128, 32, 8), 10, torch.zeros(1, dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32),
                             torch.arange(10, dtype=torch.int32)[None], torch.tensor([3], dtype=torch.int32), n_sm=0)
