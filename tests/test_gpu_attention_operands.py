"""Queries and results that attention's plain and shared plans do not take are refused before anything is launched: one that is
too small would be read or written behind its end, one off its alignment stored to where the device does not store."""
import pytest
import torch

import paper_2511_07423_b200 as syn
from test_gpu_shared import check, reference, setup as batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", [1, 2, 3, 4])
def test_results_that_cannot_be_stored_to_are_refused(kernel):
    model, kv, shared, pool, q, table, ctx, off = batch([50] * 4, [3] * 4, [(64, 4)], 64, 16, 2, seed=41)
    syn.debug_set_attention(kernel)
    try:
        plan = shared if kernel == 4 else syn.Plan(kv, torch.zeros(12, dtype=torch.int32), off, table, ctx)
    finally:
        syn.debug_set_attention(0)
    assert plan.attention_kernel() == kernel
    big = torch.full((13, q.shape[1]), 7.0, dtype=torch.float16, device="cuda")
    n = q.numel()
    bad = [big[:11], big[:12].half().float(), big[:12].cpu(), torch.empty(12, 2 * q.shape[1], dtype=torch.float16, device="cuda")[:, ::2],
           big.flatten()[1:1 + n], big.flatten()[2:2 + n]] + ([big.flatten()[4:4 + n]] if kernel == 2 else [])
    for call in (plan.attention, plan.attention_static):
        for out in bad:
            with pytest.raises(syn.SynError) as e:
                call(1, q, out)
            assert e.value.code == -1
        with pytest.raises(syn.SynError) as e:
            call(1, q[:11])
        assert e.value.code == -1
    torch.cuda.synchronize()
    assert bool((big == 7).all()) and model.status() == 0
    good = big.flatten()[8:8 + n]                                            # 16 bytes off
    plan.attention(1, q, good)
    check(good, *reference(pool, q, table, ctx, off))
    assert model.status() == 0
