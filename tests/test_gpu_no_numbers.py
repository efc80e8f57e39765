"""Keys and values that are no numbers, in attention whose results are joined from parts: they reach every row that sees them,
however many of a part's keys they are and however small that part's weight is, and no other row."""
import pytest
import torch

import paper_2511_07423_b200 as syn
from test_gpu_shared import setup as batch

pytestmark = pytest.mark.gpu

NAN = float("nan")
# chunks that leave few rows (four warps join a row's parts) and many (one warp does): more than 16 rows an SM, 2 368
FEW, MANY = [3, 1, 8, 2], [8] * 40
BATCHES = [(hd, chunk) for hd in (128, 64) for chunk in (FEW, MANY)]


def run(model, plan, q):
    out = plan.attention(1, q)
    torch.cuda.synchronize()
    assert model.status() == 0
    return out.view(q.shape[0], 8, -1)


def tokens(off, i):
    return slice(int(off[i]), int(off[i + 1]))


def agree(got, clean, hit):
    """No numbers where `hit` says so, the same bits as without them elsewhere."""
    assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("hd,chunk", BATCHES)
def test_a_shared_prefix_without_numbers(hd, chunk):
    """Every key of the prefix that all requests share: nobody's result is that of the keys behind it."""
    n = len(chunk)
    model, kv, plan, pool, q, table, ctx, off = batch([20 + i for i in range(n)], chunk, [(9, n)], hd, 8, 2, seed=11)
    assert plan.attention_kernel() == 4
    clean = run(model, plan, q)
    pool[table[0, :9].long(), 0, 0] = NAN
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[:, :4] = True
    agree(run(model, plan, q), clean, hit)


@pytest.mark.parametrize("hd,chunk", BATCHES)
def test_a_request_without_numbers_behind_its_prefix(hd, chunk):
    """Every cached key that one request has to itself (several half stages and fewer than 64 keys), among many that share with it."""
    n = len(chunk)
    for own in (30, 200):
        model, kv, plan, pool, q, table, ctx, off = batch([own] * n, chunk, [(16, n)], hd, 8, 2, seed=12)
        clean = run(model, plan, q)
        pool[table[2, 16:16 + own // 16].long(), 1, 0] = NAN
        pool[int(table[2, 16 + own // 16]), 1, 0, :own % 16] = NAN
        hit = torch.zeros_like(clean, dtype=torch.bool)
        hit[tokens(off, 2), 4:] = True
        agree(run(model, plan, q), clean, hit)


def one_key_takes_all(q, pool, table, off, hd, n):
    """All queries of a kv head alike, and one own key of each request whose score is more than 126 log2 units above every other:
    20 x the sum of |q| / sqrt(hd) x log2 e, against five standard deviations of the others at most."""
    q = q.view(-1, 2, 4, hd)
    q[:] = q[0, :, :1].clone()
    q = q.reshape(-1, 8 * hd)
    pool[:, :, 0].clamp_(-2, 2)
    top = 20 * q[0].view(2, 4, hd)[:, 0].sign()
    for i in range(n):
        pool[int(table[i, 16]), :, 0, 3] = top
    size = q[0].view(2, 4, hd)[:, 0].double().abs().sum(-1) * 1.4427 / hd ** 0.5
    assert float((20 - 2) * size.min()) > 150                  # the others: |k| <= 2 a component
    return q


@pytest.mark.parametrize("hd,chunk", BATCHES)
@pytest.mark.parametrize("which", ["key", "value"])
def test_no_number_in_a_part_of_no_weight(hd, chunk, which):
    """One such key, or one component of a value, in the shared part, whose weight is zero in 32 bits: a weight of zero times
    no number is no number, and the formula's weight is no zero."""
    n = len(chunk)
    model, kv, plan, pool, q, table, ctx, off = batch([20] * n, chunk, [(16, n)], hd, 8, 2, seed=13)
    q = one_key_takes_all(q, pool, table, off, hd, n)
    clean = run(model, plan, q)
    assert bool(clean.isfinite().all())
    hit = torch.zeros_like(clean, dtype=torch.bool)
    if which == "key":
        pool[int(table[0, 5]), 1, 0, 9, 7] = NAN
        hit[:, 4:] = True
    else:
        pool[int(table[0, 5]), 1, 1, 9, 7] = NAN
        hit[:, 4:, 7] = True
    agree(run(model, plan, q), clean, hit)


@pytest.mark.parametrize("hd", [64, 128])
def test_a_long_request_cut_into_many_parts(hd):
    """Nothing is shared; the first 64 keys, 64 in the middle, or the last page are no numbers."""
    model, kv, plan, pool, q, table, ctx, off = batch([6000], [4], [], hd, 8, 2, seed=14)
    assert plan.attention_kernel() == 4
    clean = run(model, plan, q)
    for pages in (slice(0, 4), slice(200, 204), slice(374, 375)):
        before = pool.clone()
        pool[table[0, pages].long(), 0, 0] = NAN
        hit = torch.zeros_like(clean, dtype=torch.bool)
        hit[:, :4] = True
        agree(run(model, plan, q), clean, hit)
        pool.copy_(before)
