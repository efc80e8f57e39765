"""Per-head norm, rotation and append to the paged cache (syn_op_qk_rope, syn_op_kv_append) against the formulas in 64 bits."""

import pytest
import torch

import paper_2511_07423_b200 as syn
from harness import cpu_model, to_cuda
from workloads.configs import ModelShape

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # half a step, relative
SCALINGS = {"none": dict(), "linear": dict(scaling="linear", factor=4.0), "base": dict(scaling="base", factor=8.0),
            "turns": dict(scaling="turns", factor=8.0, original_len=8192.0, low=1.0, high=4.0),
            "index": dict(scaling="index", factor=16.0, original_len=4096.0, low=1.0, high=32.0)}


def reference(x, gain, eps, rope, layout, pos):
    """(value, magnitude that the 32-bit arithmetic's error is relative to), both in 64 bits."""
    x = x.double()
    if gain is not None:
        x = x * (x.square().mean(-1, keepdim=True) + eps).rsqrt() * gain.double()
    size = x.abs()
    if rope is None:
        return x, size
    f, amp = rope.frequencies()
    h = len(f)
    ang = pos.double().cpu()[:, None] * f
    c, s = (amp * ang.cos()).to(x.device)[:, None], (amp * ang.sin()).to(x.device)[:, None]
    i = torch.arange(h, device=x.device)
    a, b = (i, i + h) if layout == "half" else (2 * i, 2 * i + 1)
    y, m = x.clone(), size.clone()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    m[..., a] = m[..., b] = amp * (size[..., a] + size[..., b])
    return y, m


def check(got, want, size):
    """One rounding to the output's type, on top of 32-bit arithmetic: a sum of up to 256 squares in 8 + 5 steps, a reciprocal
    root, three products, cosine and sine (2 units each) and two more products: below 32 units of 2^-24 of the pair."""
    clamp = want.clamp(-65504, 65504) if got.dtype == torch.float16 else want
    tol = HALF[got.dtype] * clamp.abs() + 32 * 2.0 ** -24 * size + 2.0 ** -25
    off = (got.double() - clamp).abs()
    assert bool((off <= tol).all()), float((off - tol).max())


def rows(T, heads, hd, dtype, fused, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda *s: torch.empty(*s, device="cuda", dtype=dtype).normal_(0, 1.5, generator=g)  # noqa: E731
    if fused:
        r = make(T, sum(heads), hd)
        return list(r.split(heads, 1))
    return [make(T, h, hd) for h in heads]


def gains(hd, seed):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    return [torch.empty(hd, device="cuda").normal_(1, 0.2, generator=g).to(torch.bfloat16) for _ in range(2)]


SHAPES = [   # T, q heads, k heads, head_dim, rotary
    (1, 32, 8, 128, 128), (7, 4, 2, 64, 64), (3, 5, 1, 64, 32), (33, 6, 2, 128, 54), (2, 1, 1, 8, 8), (5, 3, 3, 256, 256), (4, 7, 1, 96, 2),
    (9, 40, 8, 128, 48), (1, 3, 1, 80, 74), (300, 17, 1, 128, 128), (2, 2, 2, 16, 16), (1, 64, 64, 24, 16),
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,hq,hk,hd,rot", SHAPES)
def test_norm_and_rotation(T, hq, hk, hd, rot, dtype, layout):
    n = T + hq + rot
    scaling = sorted(SCALINGS)[n % 5]
    rope = syn.Rope(rot, 10000.0, layout, **SCALINGS[scaling])
    q, k = rows(T, [hq, hk], hd, dtype, n % 2 == 0, n)
    pos = (torch.arange(T, device="cuda", dtype=torch.int32) * 7919 * 131) % (1 << 24)
    pos[-1] = -5
    gq, gk = gains(hd, n) if n % 3 else (None, None)
    yq, yk = syn.syn_op_qk_rope(rope, q, k, pos, gq, gk, 1e-6)
    for x, y, g in ((q, yq, gq), (k, yk, gk)):
        assert y.dtype == dtype and y.shape == x.shape
        check(y, *reference(x, g, 1e-6, rope, layout, pos))
    # half precision for the attention, whatever the input
    out = torch.empty(T, hq * hd, dtype=torch.float16, device="cuda")
    got, none = syn.syn_op_qk_rope(rope, q, None, pos, gq, q_out=out)
    assert none is None and got.data_ptr() == out.data_ptr()
    check(out.view(T, hq, hd), *reference(q, gq, 1e-5, rope, layout, pos))


@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 100), ("interleaved", 128)])
def test_in_place_and_keys_alone(layout, rot):
    rope = syn.Rope(rot, 500000.0, layout)
    row, = rows(50, [12], 128, torch.bfloat16, True, 5)
    q, k, v = row[:, :8], row[:, 8:10], row[:, 10:]
    pos = torch.arange(50, device="cuda", dtype=torch.int32)
    gq, gk = gains(128, 5)
    wq, wk, before = reference(q, gq, 1e-5, rope, layout, pos), reference(k, gk, 1e-5, rope, layout, pos), v.clone()
    syn.syn_op_qk_rope(rope, q, k, pos, gq, gk, 1e-5, q, k)
    check(q, *wq)
    check(k, *wk)
    assert torch.equal(v, before)
    _, only = syn.syn_op_qk_rope(rope, None, v, pos)
    check(only, *reference(v, None, 1e-5, rope, layout, pos))


def test_norm_without_rotation_and_rotation_of_zeros():
    q, k = rows(11, [4, 2], 64, torch.float32, False, 3)
    q[0] = 0
    gq, gk = gains(64, 3)
    yq, yk = syn.syn_op_qk_rope(None, q, k, None, gq, gk)
    check(yq, *reference(q, gq, 1e-5, None, "half", None))
    check(yk, *reference(k, gk, 1e-5, None, "half", None))
    assert bool((yq[0] == 0).all())


@pytest.mark.parametrize("offset,stride_extra", [(1, 0), (0, 1), (3, 5), (8, 8)])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("half", 30), ("interleaved", 64)])
def test_rows_off_the_vector_boundaries(offset, stride_extra, layout, rot):
    rope = syn.Rope(rot, 10000.0, layout)
    T, h, hd = 13, 3, 64
    buf = rows(1, [1], (h * hd + stride_extra) * T + offset + 16, torch.bfloat16, False, 8)[0].flatten()
    x = buf.as_strided((T, h, hd), (h * hd + stride_extra, hd, 1), offset)
    out = torch.full((T * (h * hd + stride_extra) + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
    y = out.as_strided((T, h, hd), (h * hd + stride_extra, hd, 1), offset)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 3
    syn.syn_op_qk_rope(rope, x, None, pos, q_out=y)
    check(y, *reference(x, None, 1e-5, rope, layout, pos))
    mask = torch.ones_like(out, dtype=torch.bool)
    mask.as_strided((T, h, hd), (h * hd + stride_extra, hd, 1), offset).fill_(False)
    assert bool((out[mask] == 7.0).all())      # what lies between the rows stays


def test_non_finite_values_stay_in_their_head():
    q, k = rows(4, [4, 1], 64, torch.float32, True, 9)
    pos = torch.arange(4, device="cuda", dtype=torch.int32)
    clean, _ = syn.syn_op_qk_rope(syn.Rope(64), q, k, pos)
    q[1, 2, 5], q[2, 0, 0] = float("nan"), float("inf")
    got, _ = syn.syn_op_qk_rope(syn.Rope(64), q, k, pos)
    hit = torch.zeros(4, 4, dtype=torch.bool, device="cuda")
    hit[1, 2] = hit[2, 0] = True
    assert torch.equal(got[~hit], clean[~hit])
    assert not bool(got[1, 2].isfinite().all()) and not bool(got[2, 0].isfinite().all())
    big = torch.full((1, 1, 64), 1e6, device="cuda")
    out = torch.empty(1, 64, dtype=torch.float16, device="cuda")
    syn.syn_op_qk_rope(None, big, None, None, q_out=out)
    assert bool((out == 65504).all())          # saturates, as all half precision of the library


def test_empty_batches_and_refusals():
    rope = syn.Rope(64)
    z = torch.empty(0, 4, 64, device="cuda")
    q, _ = syn.syn_op_qk_rope(rope, z, None, torch.empty(0, dtype=torch.int32, device="cuda"))
    assert q.shape == (0, 4, 64)
    x = torch.zeros(2, 4, 64, device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    bad = [
        lambda: syn.syn_op_qk_rope(rope, None, None, pos),
        lambda: syn.syn_op_qk_rope(rope, x.double(), None, pos),
        lambda: syn.syn_op_qk_rope(rope, x, None, pos.long()),
        lambda: syn.syn_op_qk_rope(rope, x, None, pos[:1]),
        lambda: syn.syn_op_qk_rope(rope, x, None, pos.cpu()),
        lambda: syn.syn_op_qk_rope(rope, x, None, None),
        lambda: syn.syn_op_qk_rope(rope, x.cpu(), None, pos),
        lambda: syn.syn_op_qk_rope(rope, x, x.half(), pos),
        lambda: syn.syn_op_qk_rope(rope, x, x[:, :, :32], pos),
        lambda: syn.syn_op_qk_rope(rope, x.transpose(1, 2).contiguous().transpose(1, 2), None, pos),
        lambda: syn.syn_op_qk_rope(rope, x[:, :, :32], None, pos),
        lambda: syn.syn_op_qk_rope(rope, x[:1].expand(2, 4, 64), None, pos),
        lambda: syn.syn_op_qk_rope(rope, x, None, pos, q_gain=torch.ones(64, device="cuda")),
        lambda: syn.syn_op_qk_rope(rope, x, None, pos, q_out=torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")),
        lambda: syn.syn_op_qk_rope(rope, x, None, pos, q_out=torch.empty(2, 4, 32, device="cuda")),
        lambda: syn.syn_op_qk_rope(rope, x, x, pos, q_out=torch.empty_like(x), k_out=x.half()),
        lambda: syn.syn_op_qk_rope(syn.Rope(128), x, None, pos),
    ]
    for call in bad:
        with pytest.raises(syn.SynError) as e:
            call()
        assert e.value.code == -1


def test_another_stream_and_a_captured_graph():
    rope = syn.Rope(128, layout="interleaved")
    q, k = rows(19, [8, 2], 128, torch.bfloat16, True, 4)
    pos = torch.arange(19, device="cuda", dtype=torch.int32)
    oq, ok = torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        syn.syn_op_qk_rope(rope, q, k, pos, q_out=oq, k_out=ok)
    for seed in (1, 2):
        q.copy_(rows(19, [8], 128, torch.bfloat16, False, seed)[0])
        g.replay()
        torch.cuda.synchronize()
        check(oq, *reference(q, None, 1e-5, rope, "interleaved", pos))
        check(ok, *reference(k, None, 1e-5, rope, "interleaved", pos))
    syn.syn_op_qk_rope(rope, q, k, pos, q_out=oq.zero_(), k_out=ok, stream=torch.cuda.current_stream())
    check(oq, *reference(q, None, 1e-5, rope, "interleaved", pos))


# ------------------------------------------------------------------------------------------ append

_CACHE = {}


def model_of(hd, hq, hkv):
    if (hd, hq, hkv) not in _CACHE:
        shape = ModelShape("append", 2, 128, hq, hkv, hd, 128, 128, rms_eps=1e-5)
        _CACHE[hd, hq, hkv] = syn.Model(shape, *to_cuda(*cpu_model(shape, 1)))
    return _CACHE[hd, hq, hkv]


def batch(ctx, chunk, extra=2, seed=0):
    used = [-(-(c + n) // 16) for c, n in zip(ctx, chunk)]
    ids = torch.randperm(sum(used) + extra, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(ctx), max(used)), -9, dtype=torch.int32)
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = ids[at:at + u]
        at += u
    off = torch.tensor([0] + list(chunk)).cumsum(0).to(torch.int32)
    pos = torch.cat([torch.arange(c, c + n) for c, n in zip(ctx, chunk)])
    req = torch.repeat_interleave(torch.arange(len(ctx)), torch.tensor(chunk))
    page = table[req, pos // 16].long()
    return table, off, sum(used) + extra, pos, page


APPEND = [   # head_dim, Hq, Hkv, contexts, chunks
    (64, 4, 2, [0], [1]), (128, 8, 2, [15, 16, 0, 100], [1, 32, 17, 5]), (128, 5, 1, [1, 31], [3, 2]), (64, 16, 2, [7] * 20, [9] * 20),
    (64, 6, 2, [40], [32]),
]


@pytest.mark.parametrize("layout,rot", [("half", 0), ("half", 64), ("half", 22), ("interleaved", 64), ("interleaved", 6)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("hd,hq,hkv,ctx,chunk", APPEND)
def test_append(hd, hq, hkv, ctx, chunk, dtype, layout, rot):
    model = model_of(hd, hq, hkv)
    table, off, n_pages, pos, page = batch(ctx, chunk, seed=rot)
    kv = syn.KVCache(model, n_pages)
    T = int(off[-1])
    plan = syn.Plan(kv, torch.zeros(T, dtype=torch.int32), off, table, torch.tensor(ctx, dtype=torch.int32))
    rope = syn.Rope(rot, 10000.0, layout) if rot else None
    q, k, v = rows(T, [hq, hkv, hkv], hd, dtype, rot % 4 == 0, T + rot)
    v[0, 0, 0] = 1e5 if dtype != torch.float16 else 6e4    # beyond half precision: saturates
    gq, gk = gains(hd, T) if rot != 64 else (None, None)
    pools = [kv.layer_view(i) for i in range(2)]
    for p in pools:
        p.normal_(0, 1)
    before = [p.clone() for p in pools]
    out = plan.append(1, k, v, rope, gk, q, gq)
    torch.cuda.synchronize()
    assert torch.equal(pools[0], before[0])
    wk, wq = reference(k, gk, 1e-5, rope, layout, pos), reference(q, gq, 1e-5, rope, layout, pos)
    check(pools[1][page, :, 0, pos % 16], *wk)
    assert torch.equal(pools[1][page, :, 1, pos % 16], v.float().clamp(-65504, 65504).half())
    check(out.view(T, hq, hd), *wq)
    rest = torch.ones(n_pages, 16, dtype=torch.bool)
    rest[page, pos % 16] = False
    at, row = rest.nonzero(as_tuple=True)
    assert torch.equal(pools[1][at, :, :, row], before[1][at, :, :, row])   # every other row as it was
    # the same without queries
    pools[1].copy_(before[1])
    assert plan.append(1, k, v, rope, gk) is None
    check(pools[1][page, :, 0, pos % 16], *wk)


def test_import_and_append_agree_with_the_views():
    model = model_of(128, 8, 2)
    table, off, n_pages, pos, page = batch([20], [12])
    kv = syn.KVCache(model, n_pages)
    plan = syn.Plan(kv, torch.zeros(12, dtype=torch.int32), off, table, torch.tensor([20], dtype=torch.int32))
    k, v = rows(12, [2, 2], 128, torch.bfloat16, False, 2)
    plan.append(0, k, v)
    ek, ev = kv.export_kv(0, table[0], 20, 12)
    assert torch.equal(ek, k) and torch.equal(ev, v)
    kv.import_kv(1, table[0], 20, k, v)
    assert torch.equal(kv.layer_view(0), kv.layer_view(1))
    view = kv.layer_view(0)
    del kv, plan                                   # the view keeps the cache
    import gc
    gc.collect()
    assert bool(view.isfinite().all())


def test_append_refusals():
    model = model_of(64, 4, 2)
    table, off, n_pages, _, _ = batch([3], [2])
    kv, other = syn.KVCache(model, n_pages), syn.KVCache(model, n_pages)
    plan = syn.Plan(kv, torch.zeros(2, dtype=torch.int32), off, table, torch.tensor([3], dtype=torch.int32))
    q, k, v = rows(2, [4, 2, 2], 64, torch.bfloat16, True, 1)
    before = kv.layer_view(0).clone()
    bad = [lambda: plan.append(2, k, v), lambda: plan.append(0, q, v), lambda: plan.append(0, k[:1], v), lambda: plan.append(0, k, v.half()),
           lambda: plan.append(0, k, v, syn.Rope(66)), lambda: plan.append(0, k, v, q=k), lambda: plan.append(0, k.double(), v.double()),
           lambda: plan.append(0, k, v, q=q, q_out=torch.empty(2, 256, device="cuda")), lambda: plan.append(0, k.cpu(), v.cpu())]
    for call in bad:
        with pytest.raises(syn.SynError) as e:
            call()
        assert e.value.code == -1
    plan.kv = other                                # a plan belongs to its cache
    with pytest.raises(syn.SynError):
        plan.append(0, k, v)
    assert torch.equal(kv.layer_view(0), before)
