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
