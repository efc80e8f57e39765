"""Deeply nested prefixes: every request shares 128 keys more with the next than the one before it did.  A plan's partial rows stay within
the bound that the header states, whatever the tree, and its tokens still meet every key once."""
import pytest
import torch

import paper_2511_07423_b200 as syn
from test_shared_plan_host import shape


def staircase(n, step=8, own=3):
    """Request i's table begins with the same step * (i + 1) pages as those behind it; (tables, ctx lens, pages)."""
    table = torch.zeros(n, step * n + 2, dtype=torch.int32)
    for i in range(n):
        k = step * (i + 1)
        table[i, :k] = torch.arange(k, dtype=torch.int32)
        table[i, k:k + 2] = step * n + 2 * i + torch.arange(2, dtype=torch.int32)
    return table, torch.tensor([16 * step * (i + 1) + own for i in range(n)], dtype=torch.int32), step * n + 2 * n


@pytest.mark.parametrize("n,chunk,heads", [(16, 8, (128, 32, 8)), (64, 8, (128, 32, 8)), (256, 8, (128, 32, 8)), (200, 13, (64, 14, 2)), (512, 8, (64, 32, 8))])
def test_partial_rows_of_nested_prefixes_are_bounded(n, chunk, heads):
    hd, hq, hkv = heads
    G, T = hq // hkv, n * chunk
    table, ctx, n_pages = staircase(n)
    p = syn.plan_shared_host(shape(*heads), n_pages, torch.zeros(T, dtype=torch.int32), torch.arange(n + 1, dtype=torch.int32) * chunk, table, ctx)
    it = p["items"].long()
    rows = it[:, 7] + it[:, 1] * G * torch.where(it[:, 8] == 3, 2, 1)
    assert int(rows.max()) <= max(1 << 19, 8 * T * hq)
    assert bool((it[:, 6] < 0).any())                        # and what they share is still met together
    # keys that a token meets, counted: the item's, or those up to its own position
    met = torch.zeros(hkv, T, dtype=torch.int64)
    for q_tok, n_tok, h, req, b, e, q0, base, mode in it.tolist():
        last = torch.full((n_tok,), e) if q0 < 0 else (q0 + 1 + torch.arange(n_tok)).clamp(max=e)
        met[h, q_tok:q_tok + n_tok] += (last - b).clamp(min=0)
        if h == 0:                                             # through a table that begins with the same pages as every token's own
            first, end = q_tok // chunk, (q_tok + n_tok - 1) // chunk
            pages = -(-e // 16)
            assert bool((table[first:end + 1, b // 16:pages] == table[req, b // 16:pages]).all())
    want = ctx.long().repeat_interleave(chunk) + 1 + torch.arange(chunk).repeat(n)
    assert bool((met == want).all())


def test_prefixes_that_stay_within_the_bound_are_cut_as_finely_as_before():
    table, ctx, n_pages = staircase(16)
    p = syn.plan_shared_host(shape(128, 32, 8), n_pages, torch.zeros(128, dtype=torch.int32), torch.arange(17, dtype=torch.int32) * 8, table, ctx)
    shared = {(r[4], r[5]) for r in p["items"].tolist() if r[6] < 0}
    assert {(128 * i, 128 * (i + 1)) for i in range(1, 15)} <= shared     # (the first level's 128 keys are met by all)


@pytest.mark.parametrize("n,chunk,taken", [(32, 8, False), (64, 24, False), (64, 8, True), (128, 8, True), (64, 1, True)])
def test_what_the_merge_costs_counts(n, chunk, taken):
    """32 requests of 8 tokens leave 143 104 partial rows for 8 192 rows of output: measured 62 us against the plain kernels' 48; 64 of 24
    tokens 222 against 173.  Single tokens leave few rows, and on the coarser trees of larger batches sharing pays."""
    table, ctx, n_pages = staircase(n)
    p = syn.plan_shared_host(shape(128, 32, 8), n_pages, torch.zeros(n * chunk, dtype=torch.int32), torch.arange(n + 1, dtype=torch.int32) * chunk, table, ctx)
    assert p["taken"] == taken
