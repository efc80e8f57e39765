"""The same of the kernels in which every request reads its own keys."""
import pytest
import torch

import paper_2511_07423_b200 as syn
from test_gpu_no_numbers import NAN, agree, run, tokens
from test_gpu_shared import setup as batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kernel", [1, 2, 3])
@pytest.mark.parametrize("own,pages", [([150, 40, 700], (0, 4)), ([150, 40, 700], (4, 8)), ([150, 40, 700], (8, 10)), ([130, 40, 700], (8, 9)),
                                       ([70, 40, 700], (4, 5)), ([6000], (0, 4)), ([6000], (200, 204))])
def test_keys_without_numbers_reach_the_rows_that_see_them(own, pages, kernel, hd):
    """Whole stages of one request's keys (a stage of the tcgen05 kernel is one of its two groups' of warps)."""
    chunk = [4] * len(own)
    model, kv, _, pool, q, table, ctx, off = batch(own, chunk, [], hd, 8, 2, seed=15)
    syn.debug_set_attention(kernel)
    try:
        plan = syn.Plan(kv, torch.zeros(int(off[-1]), dtype=torch.int32), off, table, ctx)
    finally:
        syn.debug_set_attention(0)
    assert plan.attention_kernel() == kernel
    clean = run(model, plan, q)
    pool[table[0, pages[0]:pages[1]].long(), 0, 0] = NAN
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[tokens(off, 0), :4] = True
    agree(run(model, plan, q), clean, hit)
