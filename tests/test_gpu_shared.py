"""Attention over shared prefixes (plans of syn_plan_create_shared) against the formula in 64 bits, and in the step."""
import random

import pytest
import torch

import paper_2511_07423_b200 as syn
from harness import cpu_model, to_cuda
from test_shared_plan_host import tree_batch
from workloads.configs import ModelShape

pytestmark = pytest.mark.gpu

_MODELS = {}


def model_of(hd, hq, hkv, layers=2):
    if (hd, hq, hkv) not in _MODELS:
        shape = ModelShape("shared", layers, 128, hq, hkv, hd, 128, 256)
        _MODELS[hd, hq, hkv] = syn.Model(shape, *to_cuda(*cpu_model(shape, 1)))
    return _MODELS[hd, hq, hkv]


def reference(pool, q, table, ctx, off):
    """(out, sum of weights times |v|), float64 [T, Hq, hd]."""
    hkv, hd = pool.shape[1], pool.shape[4]
    hq = q.shape[1] // hd
    out = torch.empty(q.shape[0], hq, hd, dtype=torch.float64, device="cuda")
    size = torch.empty_like(out)
    for i, c in enumerate(ctx.tolist()):
        a, b = int(off[i]), int(off[i + 1])
        n = b - a
        pages = pool[table[i, :-(-(c + n) // 16)].long().cuda()].double()
        k, v = (pages[:, :, x].transpose(0, 1).reshape(hkv, -1, hd)[:, :c + n] for x in range(2))
        s = torch.einsum("nhgd,hkd->nhgk", q[a:b].double().view(n, hkv, hq // hkv, hd), k) / hd ** 0.5
        keep = torch.ones(n, c + n, dtype=torch.bool, device="cuda").tril(c)
        p = torch.where(keep[:, None, None], s, -torch.inf).softmax(-1)
        out[a:b] = torch.einsum("nhgk,hkd->nhgd", p, v).reshape(n, hq, hd)
        size[a:b] = torch.einsum("nhgk,hkd->nhgd", p, v.abs()).reshape(n, hq, hd)
    return out, size


def check(got, want, size):
    """The result's rounding to half precision (2^-11), that of every weight (2^-11), and 2^-14 of the weights for the 32-bit
    scores (a sum of hd exact products, of magnitude below 40 here: 40 * 128 * 2^-24 / sqrt(hd) at most) and exponentials."""
    got = got.double().view(want.shape)
    off = (got - want).abs()
    tol = 2.0 ** -11 * want.abs() + (2.0 ** -11 + 2.0 ** -14) * size + 2.0 ** -25
    assert bool((off <= tol).all()), (float((off / tol).max()), (off > tol).nonzero()[:5].tolist())


def setup(own, chunk, levels, hd, hq, hkv, seed=0, layer=1, q_std=1.3, force=True):
    rng = random.Random(seed)
    table, ctx, off, n_pages = tree_batch(rng, own, chunk, levels)
    model = model_of(hd, hq, hkv)
    kv = syn.KVCache(model, n_pages + 2)
    g = torch.Generator(device="cuda").manual_seed(seed)
    pool = kv.layer_view(layer)
    pool.normal_(0, 1, generator=g)
    T = int(off[-1])
    q = torch.empty(T, hq * hd, dtype=torch.float16, device="cuda").normal_(0, q_std, generator=g)
    syn.debug_set_attention(4 if force else 0)
    try:
        plan = syn.Plan(kv, torch.zeros(T, dtype=torch.int32), off, table, ctx, share_prefix=True)
    finally:
        syn.debug_set_attention(0)
    return model, kv, plan, pool, q, table, ctx, off


CASES = [   # own cached tokens, chunks, levels of (pages, group), (hd, hq, hkv)
    ([3], [1], [], (128, 8, 2)),                                       # one request, one token, one stage
    ([0], [1], [], (64, 4, 2)),                                        # its own key alone
    ([130], [5], [], (128, 8, 2)),                                     # two stages: both groups of warps
    ([500, 1300], [32, 17], [], (128, 10, 2)),                         # nothing shared, several parts a request
    ([5, 0, 40], [1, 1, 1], [(20, 3)], (128, 8, 2)),
    ([0] * 9, [32] * 9, [(8, 9)], (64, 16, 2)),                        # two tiles a leaf: 32 tokens of 8 heads
    ([100, 7, 300, 17, 90, 1], [3, 9, 1, 32, 2, 8], [(64, 6), (9, 2)], (128, 10, 2)),
    ([1] * 40, [7] * 40, [(33, 40), (12, 5), (8, 1)], (128, 6, 2)),    # two tiles of 42 tokens, odd groups of heads
    ([2] * 33, [1, 2, 3] * 11, [(300, 33), (40, 11)], (128, 7, 1)),
    ([9] * 64, [1] * 64, [(90, 64)], (128, 8, 8)),                     # one query head to a kv head: 128 tokens a tile
    ([15, 16, 17, 31, 32, 0], [1, 16, 15, 1, 32, 17], [(17, 6)], (64, 10, 2)),   # ends at, before and behind page borders
    ([20] * 50, [4] * 50, [(520, 50)], (64, 32, 8)),
    ([60] * 16, [16] * 16, [(1000, 16)], (128, 32, 8)),
]


@pytest.mark.parametrize("own,chunk,levels,heads", CASES)
def test_matches_the_formula(own, chunk, levels, heads):
    model, kv, plan, pool, q, table, ctx, off = setup(own, chunk, levels, *heads)
    assert plan.attention_kernel() == 4
    want, size = reference(pool, q, table, ctx, off)
    out = torch.full_like(q, float("nan"))
    plan.attention(1, q, out)
    torch.cuda.synchronize()
    assert model.status() == 0
    check(out, want, size)
    again = plan.attention_static(1, q)
    assert torch.equal(out, again)                    # and the same bits every time
    assert model.status() == 0


@pytest.mark.parametrize("own,chunk,heads", [([4149], [8], (128, 14, 2)), ([10460], [8], (128, 8, 1)), ([7818], [8], (64, 4, 2)),
                                             ([29589, 12000], [16, 5], (128, 14, 2))])
def test_a_few_long_requests_are_cut_finer(own, chunk, heads):
    """Nothing is shared, and the planner takes the kernel of shared prefixes by itself."""
    model, kv, plan, pool, q, table, ctx, off = setup(own, chunk, [], *heads, force=False)
    assert plan.attention_kernel() == 4
    want, size = reference(pool, q, table, ctx, off)
    check(plan.attention(1, q), want, size)
    assert model.status() == 0


def test_values_behind_a_request_do_not_reach_it():
    """Whatever lies behind the last token of a request, in its own last page and in pages it never reaches: infinities and no
    numbers, in K and in V.  Chunks end at every place of a page."""
    own, chunk = [3 * i for i in range(18)], [1 + i % 9 for i in range(18)]
    for hd, hq, hkv in ((128, 8, 2), (64, 8, 2)):
        model, kv, plan, pool, q, table, ctx, off = setup(own, chunk, [(10, 18)], hd, hq, hkv, seed=3)
        want, size = reference(pool, q, table, ctx, off)
        seen = torch.zeros(pool.shape[0], 16, dtype=torch.bool, device="cuda")
        for i in range(len(own)):
            p = torch.arange(int(ctx[i]) + chunk[i])
            seen[table[i].long().cuda()[p.cuda() // 16], p.cuda() % 16] = True
        bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda", dtype=torch.float16)
        at = (~seen).nonzero(as_tuple=True)
        pool[at[0], :, :, at[1]] = bad[torch.arange(len(at[0]), device="cuda") % 3][:, None, None, None].expand(-1, hkv, 2, hd)
        check(plan.attention(1, q), want, size)
        assert model.status() == 0


def test_no_number_in_a_key_reaches_the_rows_that_see_it():
    model, kv, plan, pool, q, table, ctx, off = setup([20, 40, 60], [3, 3, 3], [(9, 3)], 128, 8, 2, seed=4)
    clean = plan.attention(1, q)
    pool[int(table[1, 9 + 1]), 0, 0, 5] = float("nan")       # a key of request 1 alone, kv head 0
    got = plan.attention(1, q).view(9, 8, 128)
    hit = torch.zeros(9, 8, dtype=torch.bool, device="cuda")
    hit[3:6, :4] = True
    assert torch.equal(got[~hit], clean.view(9, 8, 128)[~hit]) and bool(got[hit].isnan().all())
    pool[int(table[0, 3]), 1, 0, 0] = float("nan")           # a shared key, kv head 1
    got = plan.attention(1, q).view(9, 8, 128)
    assert bool(got[:, 4:].isnan().all()) and bool(got[0:3, :4].isfinite().all())


@pytest.mark.parametrize("hd", [64, 128])
def test_scores_that_keep_growing_along_the_keys(hd):
    """The running maximum moves in every half stage, in one half of the query heads up and in the other down: O is rescaled in tensor
    memory all the time, and parts differ by many orders of magnitude."""
    model, kv, plan, pool, q, table, ctx, off = setup([700, 130, 1400, 9], [16, 5, 32, 1], [(70, 4)], hd, 8, 2, seed=5, q_std=0.05)
    q = q.view(-1, 8, hd)
    q[:, 0::2, 0], q[:, 1::2, 0] = 31.0, -31.0
    pool[:, :, 0] *= 0.05
    slope = 0.1 * hd ** 0.5 / (31.0 * 1.4426950408889634)     # 0.1 log2 units a key, ten times the gap at which O is rescaled in 800 keys
    for i in range(4):
        p = torch.arange(int(ctx[i]) + int(off[i + 1] - off[i]), device="cuda")
        pool[table[i].long().cuda()[p // 16], :, 0, p % 16, 0] = (slope * p).half()[:, None]
    q = q.reshape(-1, 8 * hd)
    want, size = reference(pool, q, table, ctx, off)
    got = plan.attention(1, q).double().view(want.shape)
    # scores up to 0.1 ln 2 * 2600 = 180, a relative error of 2^-24 for each of a few operations on them: 2^-14 of the weights and more
    tol = 2.0 ** -11 * want.abs() + (2.0 ** -11 + 180 * 8 * 2.0 ** -24) * size + 2.0 ** -25
    assert bool(((got - want).abs() <= tol).all())
    assert model.status() == 0


def test_equal_scores_and_one_key_that_takes_all():
    model, kv, plan, pool, q, table, ctx, off = setup([33] * 5, [2] * 5, [(40, 5)], 128, 8, 2, seed=6)
    want, size = reference(pool, torch.zeros_like(q), table, ctx, off)
    check(plan.attention(1, torch.zeros_like(q)), want, size)              # all weights equal: the mean of V
    pool[int(table[0, 7]), :, 0, 3] = 30 * q[0].view(8, 128)[0::4].sign()[:, None].reshape(2, 128)
    pool[:, :, 0] *= 0.01
    pool[int(table[0, 7]), :, 0, 3] *= 100
    want, size = reference(pool, q, table, ctx, off)
    got = plan.attention(1, q).double().view(want.shape)
    # scores in the hundreds (30 * 128 * 1.3 / 11): their 2^-24 is 2^-14 of a weight at most
    assert bool(((got - want).abs() <= 2.0 ** -11 * want.abs() + (2.0 ** -11 + 2.0 ** -13) * size + 2.0 ** -25).all())


def test_another_stream_a_captured_graph_and_two_plans():
    model, kv, plan, pool, q, table, ctx, off = setup([50] * 12, [3] * 12, [(64, 12)], 64, 16, 2, seed=7)
    T = int(off[-1])
    syn.debug_set_attention(4)
    try:
        other = syn.Plan(kv, torch.zeros(3, dtype=torch.int32), off[:2], table[:1], ctx[:1], share_prefix=True)   # another batch on the same cache
    finally:
        syn.debug_set_attention(0)
    out, out2 = torch.empty_like(q), torch.empty(3, q.shape[1], dtype=torch.float16, device="cuda")
    plan.attention(1, q, out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        plan.attention(1, q, out)
        other.attention(1, q[:3], out2)
    for seed in range(3):
        q.normal_(0, 1.2, generator=torch.Generator(device="cuda").manual_seed(seed))
        g.replay()
        torch.cuda.synchronize()
        check(out, *reference(pool, q, table, ctx, off))
        check(out2, *reference(pool, q[:3], table[:1], ctx[:1], off[:2]))
    assert model.status() == 0


def test_pages_far_into_a_large_cache():
    """Pages beyond 2^31 elements of the pool, for the append and for the attention."""
    hd, hq, hkv = 128, 8, 8
    model = model_of(hd, hq, hkv, layers=2)
    n_pages = 70000                                                          # 32 768 elements each
    kv = syn.KVCache(model, n_pages)
    pool = kv.layer_view(1)
    rng = random.Random(1)
    ids = rng.sample(range(66000, n_pages), 60)
    table = torch.tensor([ids[:20] + ids[20 + 5 * i:25 + 5 * i] for i in range(6)], dtype=torch.int32)
    ctx, chunk = torch.full((6,), 340, dtype=torch.int32), 4
    off = torch.arange(0, 7 * chunk, chunk, dtype=torch.int32)
    pool[66000:] = torch.empty(4000, hkv, 2, 16, hd, device="cuda", dtype=torch.float16).normal_(0, 1)
    syn.debug_set_attention(4)
    try:
        plan = syn.Plan(kv, torch.zeros(24, dtype=torch.int32), off, table, ctx, share_prefix=True)
    finally:
        syn.debug_set_attention(0)
    k, v = (torch.empty(24, hkv, hd, device="cuda", dtype=torch.float16).normal_(0, 1) for _ in range(2))
    plan.append(1, k, v)
    pos = 340 + torch.arange(4).repeat(6)
    page = table[torch.arange(6).repeat_interleave(4), pos // 16].long()
    assert torch.equal(pool[page, :, 0, pos % 16], k) and torch.equal(pool[page, :, 1, pos % 16], v)
    q = torch.empty(24, hq * hd, device="cuda", dtype=torch.float16).normal_(0, 1.3)
    check(plan.attention(1, q), *reference(pool, q, table, ctx, off))
    assert not bool(pool[:66000].any())


def test_projections_appended_and_attended():
    """The operators as they are used together: one fused projection row per token, norms, an interleaved rotation stretched for long contexts,
    the append, and attention of a batch that shares its prompt, against the same in 64 bits."""
    hd, hq, hkv = 128, 8, 2
    model, kv, plan, pool, _, table, ctx, off = setup([17, 80, 300, 5], [5, 1, 8, 2], [(50, 4)], hd, hq, hkv, seed=8)
    T = int(off[-1])
    g = torch.Generator(device="cuda").manual_seed(8)
    row = torch.empty(T, hq + 2 * hkv, hd, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    q, k, v = row.split([hq, hkv, hkv], 1)
    gq, gk = (torch.empty(hd, device="cuda").normal_(1, 0.1, generator=g).to(torch.bfloat16) for _ in range(2))
    rope = syn.Rope(96, 500000.0, "interleaved", scaling="turns", factor=8.0, original_len=8192.0, low=1.0, high=4.0)
    qr = plan.append(1, k, v, rope, gk, q, gq)
    out = plan.attention(1, qr)
    # dense: the same operator without a cache agrees bit for bit
    pos = torch.cat([torch.arange(int(ctx[i]), int(ctx[i]) + int(off[i + 1] - off[i])) for i in range(4)]).to(torch.int32).cuda()
    dq = torch.empty(T, hq, hd, dtype=torch.float16, device="cuda")
    dk = torch.empty(T, hkv, hd, dtype=torch.float16, device="cuda")
    syn.syn_op_qk_rope(rope, q, k, pos, gq, gk, 1e-5, dq, dk)
    assert torch.equal(dq.flatten(1), qr)
    page = torch.cat([table[i].long()[torch.arange(int(ctx[i]), int(ctx[i]) + int(off[i + 1] - off[i])) // 16] for i in range(4)])
    assert torch.equal(pool[page, :, 0, pos.cpu().long() % 16], dk) and torch.equal(pool[page, :, 1, pos.cpu().long() % 16], v.half())
    check(out, *reference(pool, qr, table, ctx, off))
    # and a plan of the plain kernels on the same batch
    plain = syn.Plan(kv, torch.zeros(T, dtype=torch.int32), off, table, ctx)
    assert plain.attention_kernel() in (1, 2, 3)
    check(plain.attention(1, qr), *reference(pool, qr, table, ctx, off))


def test_refusals():
    model, kv, plan, pool, q, table, ctx, off = setup([50] * 4, [3] * 4, [(64, 4)], 64, 16, 2)
    before = pool.clone()
    with pytest.raises(syn.SynError):
        plan.attention(2, q)
    shifted = torch.empty(q.numel() + 8, dtype=torch.float16, device="cuda")[4:4 + q.numel()].view_as(q)
    with pytest.raises(syn.SynError) as e:
        plan.attention(1, shifted)                            # 8 bytes off: the tile loads need 16
    assert e.value.code == -1
    other = syn.KVCache(model, kv.n_pages)
    plan.kv = other
    with pytest.raises(syn.SynError):
        plan.attention(1, q)
    plan.kv = kv
    bad = table.clone()
    bad[1, 3] = kv.n_pages
    with pytest.raises(syn.SynError) as e:
        syn.Plan(kv, torch.zeros(12, dtype=torch.int32), off, bad, ctx, share_prefix=True)
    assert e.value.code == -4
    bad = table.clone()
    bad[1] = bad[0]                                           # two chunks on the same slots
    with pytest.raises(syn.SynError) as e:
        syn.Plan(kv, torch.zeros(12, dtype=torch.int32), off, bad, ctx, share_prefix=True)
    assert e.value.code == -7
    assert torch.equal(pool, before) and model.status() == 0


def test_the_step_over_shared_prefixes():
    """syn_verify_run on a shared plan against a plain plan of the same batch.  Either is within 0.03 standard deviations of the exact logits
    (the bound of the step's own tests), so they are within 0.06 of each other, and argmaxes with twice that gap agree."""
    shape = ModelShape("shared-step", 3, 256, 8, 2, 64, 512, 1024)
    model = syn.Model(shape, *to_cuda(*cpu_model(shape, 3)))
    rng = random.Random(3)
    own, chunk = [rng.randint(0, 90) for _ in range(20)], [rng.randint(1, 9) for _ in range(20)]
    table, ctx, off, n_pages = tree_batch(rng, own, chunk, [(12, 20), (8, 5)])
    T = int(off[-1])
    tok = torch.randint(0, 1024, (T,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    got = []
    for share in (False, True):
        kv = syn.KVCache(model, n_pages)
        for layer in range(3):
            kv.layer_view(layer).normal_(0, 0.5, generator=torch.Generator(device="cuda").manual_seed(layer))
        syn.debug_set_attention(4)
        try:
            plan = syn.Plan(kv, tok, off, table, ctx, share_prefix=share)
        finally:
            syn.debug_set_attention(0)
        assert (plan.attention_kernel() == 4) == share
        acc, cor = (torch.full((20,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
        top1 = torch.empty(T, dtype=torch.int32, device="cuda")
        logits = torch.empty(T, 1024, device="cuda")
        model.set_profile(True)
        plan.run(acc, cor, top1, logits)
        prof = model.get_profile()
        model.set_profile(False)
        assert model.status() == 0
        assert prof["attention"][1] == 3 and prof["attention_merge"][1] == (3 if share else 0)
        assert sum(n for _, n in prof.values()) == plan.stats().kernel_launches
        got.append((logits, top1, acc, cor, kv.layer_view(2).clone()))
    (la, ta, aa, ca, pa), (lb, tb, ab, cb, pb) = got
    sigma = float(la.std())
    assert float((la - lb).abs().max()) <= 0.06 * sigma
    two = la.topk(2).values
    clear = (two[:, 0] - two[:, 1]) > 0.12 * sigma
    assert torch.equal(ta[clear], tb[clear]) and bool(clear.any())
    assert float((pa.float() - pb.float()).abs().max()) <= 0.06 * float(pa.float().std())


def test_without_room_for_partials_the_batch_is_planned_as_ever():
    own, chunk, levels = [60] * 32, [32] * 32, [(300, 32)]                   # 60 MB of partials and more
    model, kv, plan, pool, q, table, ctx, off = setup(own, chunk, levels, 128, 32, 8, force=False)
    T = int(off[-1])
    assert plan.attention_kernel() == 4
    want = plan.attention(1, q)
    plain = syn.Plan(kv, torch.zeros(T, dtype=torch.int32), off, table, ctx)   # (the model's workspaces are there)
    plan.close()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    fill = torch.empty(torch.cuda.mem_get_info()[0] - (16 << 20), dtype=torch.uint8, device="cuda")
    assert torch.cuda.mem_get_info()[0] < 24 << 20                           # the plan's lists fit, its partials do not
    again = syn.Plan(kv, torch.zeros(T, dtype=torch.int32), off, table, ctx, share_prefix=True)
    assert again.attention_kernel() == plain.attention_kernel() != 4
    del fill
    torch.cuda.empty_cache()
    got = again.attention(1, q)
    size = pool.abs().max().double()
    # two results of the same formula, each within 2^-11 of the weights and of the value
    assert float((got.double() - want.double()).abs().max()) <= float(2 * (2 * 2.0 ** -11 + 2.0 ** -14) * size)
    assert model.status() == 0
