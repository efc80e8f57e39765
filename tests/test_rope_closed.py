"""A rotation that was closed is refused: the library's null handle stands for no rotation at all, and unrotated keys would enter the cache."""
import pytest
import torch

import paper_2511_07423_b200 as syn


def closed():
    rope = syn.Rope(64)
    rope.close()
    return rope


def test_a_closed_rotation_is_refused():
    x = torch.zeros(2, 4, 64)
    for q, k in ((x, None), (None, x), (x, x), (x[:0], None)):
        with pytest.raises(syn.SynError) as e:
            syn.syn_op_qk_rope(closed(), q, k, torch.zeros(len(x), dtype=torch.int32))
        assert e.value.code == -1 and "closed" in str(e.value)
    with pytest.raises(syn.SynError):
        closed().frequencies()


@pytest.mark.gpu
def test_a_closed_rotation_is_refused_by_the_append_and_nothing_is_written():
    from test_gpu_rope import batch, model_of, rows
    model = model_of(64, 4, 2)
    table, off, n_pages, _, _ = batch([3], [2])
    kv = syn.KVCache(model, n_pages)
    plan = syn.Plan(kv, torch.zeros(2, dtype=torch.int32), off, table, torch.tensor([3], dtype=torch.int32))
    q, k, v = rows(2, [4, 2, 2], 64, torch.bfloat16, True, 1)
    before = kv.layer_view(0).clone()
    with pytest.raises(syn.SynError) as e:
        plan.append(0, k, v, closed(), q=q)
    assert e.value.code == -1 and "closed" in str(e.value)
    q0 = q.clone()
    with pytest.raises(syn.SynError):
        syn.syn_op_qk_rope(closed(), q, None, torch.zeros(2, dtype=torch.int32, device="cuda"), q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(kv.layer_view(0), before) and torch.equal(q, q0)
