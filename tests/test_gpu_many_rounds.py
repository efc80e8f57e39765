"""Loops that only large batches enter: warps of the rotation that take several rounds of heads, and merges that join more parts of a row
than a warp fetches at a time."""
import pytest
import torch

import paper_2511_07423_b200 as syn
from test_gpu_rope import batch, check, gains, model_of, reference, rows
from test_gpu_shared import check as check_attention, model_of as attention_model, reference as attention_reference, setup
from test_shared_plan_rows import staircase

pytestmark = pytest.mark.gpu


def rounds(T, heads, hd):
    """Rounds of four accesses that a warp of the rotation takes where all its heads go round (148 SMs, 16 warps each)."""
    lanes = 1
    while 8 * lanes < hd:
        lanes *= 2
    per = 32 // lanes
    return min(5, T * sum(-(-h // per) for h in heads) // (148 * 16 * 4))


FORMS = [("half", 1.0, 0), ("interleaved", 1.0, 0), ("half", 0.5, 0), ("half", 54 / 128, 0), ("interleaved", 54 / 128, 0), ("half", 1.0, 1)]
SIZES = [(1000, 37, 9, 128, 2), (2600, 37, 9, 128, 5), (2300, 21, 2, 80, 2), (700, 37, 5, 256, 3)]   # the last: rounds


@pytest.mark.parametrize("layout,part,offset", FORMS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,hq,hk,hd,n_rounds", SIZES)
def test_rotation_in_several_rounds(T, hq, hk, hd, n_rounds, dtype, layout, part, offset):
    """Head counts that end within a round; rows on and off the vector boundaries; the inputs' type, half precision, and in place."""
    assert rounds(T, [hq, hk], hd) == n_rounds
    rot = int(hd * part) // 2 * 2
    rope = syn.Rope(rot, 500000.0, layout)
    buf = rows(1, [1], T * (hq + hk) * hd + 8, dtype, False, T + hd)[0].flatten()
    q, k = buf[offset:offset + T * (hq + hk) * hd].view(T, hq + hk, hd).split([hq, hk], 1)
    pos = torch.randint(0, 1 << 17, (T,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(T))
    gq, gk = gains(hd, T) if hq % 2 else (None, None)
    wq, wk = reference(q, gq, 1e-5, rope, layout, pos), reference(k, gk, 1e-5, rope, layout, pos)
    half = torch.empty(T, hq, hd, dtype=torch.float16, device="cuda"), torch.empty(T, hk, hd, dtype=torch.float16, device="cuda")
    for outs in ((None, None), half, (q, k)):                  # in place at last
        yq, yk = syn.syn_op_qk_rope(rope, q, k, pos, gq, gk, 1e-5, *outs)
        check(yq, *wq)
        check(yk, *wk)


@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 54), ("interleaved", 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_append_in_several_rounds(dtype, layout, rot):
    hd, hq, hkv, n = 128, 42, 6, 64
    chunk = [32] * (n - 1) + [19]
    assert rounds(sum(chunk), [hq, hkv, hkv], hd) == 5
    model = model_of(hd, hq, hkv)
    table, off, n_pages, pos, page = batch([3 * i for i in range(n)], chunk, seed=rot)
    kv = syn.KVCache(model, n_pages)
    T = int(off[-1])
    plan = syn.Plan(kv, torch.zeros(T, dtype=torch.int32), off, table, torch.tensor([3 * i for i in range(n)], dtype=torch.int32))
    rope = syn.Rope(rot, 10000.0, layout)
    q, k, v = rows(T, [hq, hkv, hkv], hd, dtype, True, T + rot)
    gq, gk = gains(hd, T)
    pool = kv.layer_view(1)
    pool.normal_(0, 1)
    before = pool.clone()
    out = plan.append(1, k, v, rope, gk, q, gq)
    check(out.view(T, hq, hd), *reference(q, gq, 1e-5, rope, layout, pos))
    check(pool[page, :, 0, pos % 16], *reference(k, gk, 1e-5, rope, layout, pos))
    assert torch.equal(pool[page, :, 1, pos % 16], v.half())
    rest = torch.ones(n_pages, 16, dtype=torch.bool)
    rest[page, pos % 16] = False
    at, row = rest.nonzero(as_tuple=True)
    assert torch.equal(pool[at, :, :, row], before[at, :, :, row])


@pytest.mark.parametrize("hd,hkv,chunk", [(128, 1, 3), (64, 2, 1)])
def test_a_row_of_hundreds_of_parts(hd, hkv, chunk):
    """One request of 131 072 keys, one kv head or two: a row's parts are more than four warps fetch at a time."""
    model, kv, plan, pool, q, table, ctx, off = setup([131072], [chunk], [], hd, 8, hkv, seed=31)
    shape = model.shape
    p = syn.plan_shared_host(shape, kv.n_pages, torch.zeros(chunk, dtype=torch.int32), off, table, ctx)["parts"]
    assert int((p[:, 0] == 0).sum()) > 128 * hkv
    out = plan.attention(1, q)
    # sums in 32 bits, of a thousand keys a part at most and of 74 parts a warp: some 200 additions, 2^-16 of the
    # weights, beside 2^-15 for the scores, within the tolerance's 2^-14
    want, size = attention_reference(pool, q, table, ctx, off)
    check_attention(out, want, size)
    assert torch.equal(out, plan.attention(1, q)) and model.status() == 0


def test_many_rows_of_more_than_32_parts():
    """A warp a row, and prefixes nested 40 deep."""
    n, chunk, hq, hkv, hd = 40, 8, 8, 2, 128
    table, ctx, n_pages = staircase(n)
    model = attention_model(hd, hq, hkv)
    kv = syn.KVCache(model, n_pages)
    pool = kv.layer_view(1)
    pool.normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(32))
    off = torch.arange(n + 1, dtype=torch.int32) * chunk
    T = n * chunk
    assert T * hq > 148 * 16
    p = syn.plan_shared_host(model.shape, n_pages, torch.zeros(T, dtype=torch.int32), off, table, ctx)["parts"]
    assert int((p[:, 0] == T - 1).sum()) > 32 * hkv
    q = torch.empty(T, hq * hd, dtype=torch.float16, device="cuda").normal_(0, 1.3, generator=torch.Generator(device="cuda").manual_seed(33))
    syn.debug_set_attention(4)
    try:
        plan = syn.Plan(kv, torch.zeros(T, dtype=torch.int32), off, table, ctx, share_prefix=True)
    finally:
        syn.debug_set_attention(0)
    check_attention(plan.attention(1, q), *attention_reference(pool, q, table, ctx, off))
    assert model.status() == 0
