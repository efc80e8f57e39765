"""Results of calls that are given a stream: their memory is that stream's, not what the current stream let go a moment ago and may
still be using."""
import pytest
import torch

import paper_2511_07423_b200 as syn
from test_gpu_rope import rows
from test_gpu_shared import check, reference, setup as batch

pytestmark = pytest.mark.gpu


def owner(t):
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]


def test_results_belong_to_the_stream_that_writes_them():
    model, kv, plan, pool, q, table, ctx, off = batch([40] * 9, [3] * 9, [(64, 9)], 128, 8, 2, seed=16)
    plain = syn.Plan(kv, torch.zeros(27, dtype=torch.int32), off, table, ctx)
    rope, pos = syn.Rope(128), torch.arange(27, dtype=torch.int32, device="cuda")
    qh, k, v = rows(27, [8, 2, 2], 128, torch.float16, False, 16)
    w = torch.ones(256, q.shape[1], dtype=torch.bfloat16, device="cuda")
    s, here = torch.cuda.Stream(), torch.cuda.current_stream()
    s.wait_stream(here)
    calls = [lambda st: plan.append(1, k, v, rope, q=qh, stream=st), lambda st: plan.attention(1, q, stream=st), lambda st: plan.attention_static(1, q, stream=st),
             lambda st: plain.attention(1, q, stream=st), lambda st: syn.syn_op_qk_rope(rope, qh, None, pos, stream=st)[0],
             lambda st: syn.syn_op_qk_rope(rope, None, k, pos, stream=st)[1], lambda st: syn.syn_op_linear(q, w, st),
             lambda st: kv.export_kv(1, table[0], 5, 40, st)[1],
             lambda st: kv.verify_batch(torch.zeros(27, dtype=torch.int32), off, table, ctx, want_logits=True, stream=st)[2]]
    for call in calls:
        y = call(s)
        s.synchronize()
        assert owner(y) == s.cuda_stream
        torch.cuda.synchronize()
        z = call(None)
        assert owner(z) == here.cuda_stream and torch.equal(y, z)
        torch.cuda.synchronize()
    check(plan.attention(1, q), *reference(pool, q, table, ctx, off))
    assert model.status() == 0
