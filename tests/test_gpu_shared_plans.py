"""What plans over shared prefixes hold, and what becomes of them where the planner expects no gain or the device has no room."""
import random

import pytest
import torch

import paper_2511_07423_b200 as syn
from test_gpu_shared import check, model_of, reference, setup as batch
from test_shared_plan_host import tree_batch

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
