"""What plans over shared prefixes hold, and what becomes of them where the planner expects no gain or the device has no room."""
import random

import pytest
import torch

import paper_2511_07423_b200 as syn
from test_gpu_shared import check, model_of, reference, setup as batch
from test_shared_plan_host import tree_batch
from test_shared_plan_rows import staircase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("own,chunk,levels", [([500] * 4, [2] * 4, []), ([1000] * 30, [4] * 30, [(8, 30)])])
def test_a_batch_without_gain_holds_what_a_plain_plan_holds(own, chunk, levels):
    model, kv, _, pool, q, table, ctx, off = batch(own, chunk, levels, 128, 32, 8, seed=21, force=False)
    tok = torch.zeros(int(off[-1]), dtype=torch.int32)
    plain, plan = syn.Plan(kv, tok, off, table, ctx), syn.Plan(kv, tok, off, table, ctx, share_prefix=True)
    assert plan.attention_kernel() == plain.attention_kernel() != 4
    a, b = plain.stats(), plan.stats()
    assert [(n, getattr(a, n)) for n, _ in a._fields_] == [(n, getattr(b, n)) for n, _ in b._fields_]
    assert torch.equal(plain.attention(1, q), plan.attention(1, q)) and model.status() == 0


def test_room_for_the_partials_but_not_for_the_lists():
    """Page tables of 100 000 columns: 13 MB of lists, for which the plan takes half as much again, beside 65 536 partial rows of
    520 bytes, 34 MB.  44 MB hold either, not both; what remains is a plain plan."""
    own, chunk, levels = [60] * 32, [32] * 32, [(300, 32)]
    table, ctx, off, n_pages = tree_batch(random.Random(22), own, chunk, levels)
    wide = torch.full((32, 100000), -7, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    model = model_of(128, 32, 8)
    kv = syn.KVCache(model, n_pages)
    pool = kv.layer_view(1)
    pool.normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(22))
    T = int(off[-1])
    tok = torch.zeros(T, dtype=torch.int32)
    q = torch.empty(T, 32 * 128, dtype=torch.float16, device="cuda").normal_(0, 1.3)
    want, size = reference(pool, q, table, ctx, off)
    plain = syn.Plan(kv, tok, off, wide, ctx)                      # (the model's workspaces are there)
    kernel = plain.attention_kernel()
    shared = syn.Plan(kv, tok, off, wide, ctx, share_prefix=True)
    assert shared.attention_kernel() == 4 != kernel
    plain.close()
    shared.close()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    fill = torch.empty(torch.cuda.mem_get_info()[0] - (44 << 20), dtype=torch.uint8, device="cuda")
    assert 40 << 20 <= torch.cuda.mem_get_info()[0] <= 48 << 20
    again = syn.Plan(kv, tok, off, wide, ctx, share_prefix=True)
    assert again.attention_kernel() == kernel
    assert torch.cuda.mem_get_info()[0] > 20 << 20                 # the partials have gone back
    del fill
    torch.cuda.empty_cache()
    check(again.attention(1, q), want, size)
    assert model.status() == 0


def test_nested_prefixes_on_a_coarser_tree():
    """64 requests of 8 tokens whose common prefixes grow by 128 keys from one to the next: the whole tree would leave 548 608 rows."""
    n, chunk, hq, hkv, hd = 64, 8, 32, 8, 128
    table, ctx, n_pages = staircase(n)
    model = model_of(hd, hq, hkv)
    kv = syn.KVCache(model, n_pages)
    pool = kv.layer_view(1)
    pool.normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(23))
    off = torch.arange(n + 1, dtype=torch.int32) * chunk
    q = torch.empty(n * chunk, hq * hd, dtype=torch.float16, device="cuda").normal_(0, 1.3)
    plan = syn.Plan(kv, torch.zeros(n * chunk, dtype=torch.int32), off, table, ctx, share_prefix=True)
    assert plan.attention_kernel() == 4
    check(plan.attention(1, q), *reference(pool, q, table, ctx, off))
    assert model.status() == 0
