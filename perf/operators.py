"""The measured work of the operators around a plan: rotating queries and keys, appending keys and values to the paged
cache, and the attention of batches whose requests share prefixes.

A case is a dict of plain values:
  op        "rope"    syn_op_qk_rope: per-head norm and rotation of queries and keys, dense in, dense out
            "append"  Plan.append: norm, rotation and append of a batch's keys and values, its queries in the same launch
            "prefix"  Plan(share_prefix=True).attention: attention of a batch that shares prefixes
  hq, hkv, hd         query heads, kv heads, components of a head
  rope, append: layout "half" or "interleaved", rotary components that rotate, scaling as in Rope, norm: gains are given,
            dtype of the projections' outputs; fused: q, k and v are slices of one row per token
  rope: tokens; far: largest position
  append, prefix: requests, ctx_lo..ctx_hi cached tokens behind what is shared, chunk_lo..chunk_hi tokens a request adds
  append: queries: the call rotates them too
  prefix: shared: tokens that the whole batch shares; more: tokens that every `group` neighbours share beyond those
Lengths follow from the case, contents from the seed.  The cache is half precision, [page][kv head][K, V][16][hd].
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
PAGE = 16
EPS = 1e-5
BASE = 500000.0
HALF_MAX = 65504.0
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# how the frequencies are stretched for long contexts; the fields are Rope's
SCALINGS = {
    "none": dict(scaling="none"),
    "linear": dict(scaling="linear", factor=4.0),
    "base": dict(scaling="base", factor=8.0),
    "turns": dict(scaling="turns", factor=8.0, original_len=8192.0, low=1.0, high=4.0),
    "index": dict(scaling="index", factor=16.0, original_len=4096.0, low=1.0, high=32.0),
}


def _rope(name, tokens, hq, hkv, hd, layout, rotary, scaling, norm, dtype, fused, far):
    c = dict(op="rope", tokens=tokens, hq=hq, hkv=hkv, hd=hd, layout=layout, rotary=rotary, scaling=scaling, norm=norm, dtype=dtype,
             fused=fused, far=far)
    return dict(c, name=name) if name else c


def _append(name, requests, ctx, chunk, hq, hkv, hd, layout, rotary, scaling, norm, dtype, fused, queries):
    c = dict(op="append", requests=requests, ctx_lo=ctx[0], ctx_hi=ctx[1], chunk_lo=chunk[0], chunk_hi=chunk[1], hq=hq, hkv=hkv, hd=hd,
             layout=layout, rotary=rotary, scaling=scaling, norm=norm, dtype=dtype, fused=fused, queries=queries)
    return dict(c, name=name) if name else c


def _prefix(name, requests, shared, more, group, ctx, chunk, hq, hkv, hd):
    c = dict(op="prefix", requests=requests, shared=shared, more=more, group=group, ctx_lo=ctx[0], ctx_hi=ctx[1], chunk_lo=chunk[0],
             chunk_hi=chunk[1], hq=hq, hkv=hkv, hd=hd)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one request on the 8B heads: what a lone decode step waits for
        _rope("rope-8b-one", 1, 32, 8, 128, "half", 128, "none", True, "bf16", True, 4000),
        # an ordinary verification batch of the 1B heads, a quarter of each head rotates, neighbours paired, no norm
        _rope("rope-1b-batch", 181, 32, 8, 64, "interleaved", 16, "linear", False, "fp16", True, 2048),
        # a large prefill, norms and stretched frequencies, positions of a very long document
        _rope("rope-8b-prefill", 8192, 32, 8, 128, "half", 128, "turns", True, "bf16", False, 1 << 20),
        # one token of one request of the 1B heads enters the cache
        _append("append-1b-one", 1, (777, 777), (1, 1), 32, 8, 64, "half", 64, "none", False, "bf16", True, True),
        # the benchmark's batch: 64 devices, chunks of 1 to 16, fused projection output
        _append("append-8b-64", 64, (100, 400), (1, 16), 32, 8, 128, "half", 128, "turns", True, "bf16", True, True),
        # chunked prefill of many requests, keys and values alone, fp32 from an adapter's sum, half of each head rotates
        _append("append-8b-256x32", 256, (0, 150), (32, 32), 32, 8, 128, "interleaved", 64, "index", True, "fp32", False, False),
        # four devices under one system prompt on the 1B heads
        _prefix("prefix-1b-4", 4, 1024, 0, 1, (1, 80), (1, 1), 32, 8, 64),
        # three requests, one token each, on one very long document: the keys' bytes count
        _prefix("prefix-8b-long-3", 3, 131072, 0, 1, (5, 300), (1, 1), 32, 8, 128),
        # the benchmark's batch behind a long instruction, own dialogues of some hundred tokens
        _prefix("prefix-8b-64", 64, 4096, 0, 1, (30, 700), (1, 16), 32, 8, 128),
        # two levels: a system prompt for all, a document for each eight neighbours; five query heads to a kv head
        _prefix("prefix-32b-two-levels", 72, 2000, 1100, 8, (10, 400), (1, 9), 40, 8, 128),
        # 32-token chunks of prompts over one shared document
        _prefix("prefix-8b-24x32", 24, 32768, 0, 1, (0, 900), (32, 32), 32, 8, 128),
        # the largest: 256 devices, eight tokens each, on a document whose length is no multiple of a tile
        _prefix("prefix-8b-256", 256, 12016, 0, 1, (20, 200), (8, 8), 32, 8, 128),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rope", "append", "prefix", "prefix"))
    hq, hkv, hd = rng.choice(((32, 8, 64), (32, 8, 128), (40, 8, 128), (4, 2, 64), (8, 1, 128), (6, 2, 64), (14, 2, 128), (8, 8, 128)))
    if op != "prefix":
        layout = rng.choice(("half", "interleaved"))
        rotary = 2 * rng.randint(1, hd // 2) if rng.random() < 0.5 else hd
        scaling = rng.choice(sorted(SCALINGS))
        norm, fused = rng.random() < 0.5, rng.random() < 0.5
        dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if op == "rope":
        return _rope(None, _log(rng, 1, 3400 if dtype == "fp32" else 6800), hq, hkv, hd, layout, rotary, scaling, norm, dtype, fused, _log(rng, 64, 1 << 20))
    if op == "append":
        lo = rng.randint(0, 120)
        chunk = rng.choice(((1, 1), (1, rng.randint(2, 16)), (32, 32), (17, 32)))
        return _append(None, _log(rng, 1, 200), (lo, lo + rng.randint(0, 60)), chunk, hq, hkv, hd, layout, rotary, scaling, norm, dtype,
                       fused, rng.random() < 0.6)
    while True:
        requests, shared = _log(rng, 1, 256), _log(rng, 16, 65536)
        more, group = (_log(rng, 16, 4096), rng.randint(2, 16)) if rng.random() < 0.3 else (0, 1)
        lo = _log(rng, 1, 500)
        chunk = rng.choice(((1, 1), (1, rng.randint(2, 16)), (rng.randint(2, 8),) * 2, (17, 32), (32, 32)))
        c = _prefix(None, requests, shared, more, group, (lo, lo + _log(rng, 1, 1000)), chunk, hq, hkv, hd)
        keys = shared + more + c["ctx_hi"] + chunk[1]
        # no more arithmetic than the largest listed case, and room for the plain form's copy of every request's keys
        if requests * chunk[1] * hq * hd * keys < 256 * 8 * 32 * 128 * 12016 and requests * keys * hkv * hd < 256 * 12300 * 8 * 128:
            return c


# ------------------------------------------------------------------------------------------ what a case is made of

def _lengths(case):
    """Tokens that request i shares with its neighbours, its cached tokens (those included) and its chunk."""
    rng = random.Random("/".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))
    ctx = [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["requests"])]
    chunk = [rng.randint(case["chunk_lo"], case["chunk_hi"]) for _ in ctx]
    common = (case.get("shared", 0) + PAGE - 1) // PAGE * PAGE if case.get("shared") else 0
    more = (case["more"] + PAGE - 1) // PAGE * PAGE if case.get("more") else 0
    return common, more, [common + more + c for c in ctx], chunk


def _tables(case, np_rng):
    """Page tables [requests, most pages] of a batch, the pages of the pool and its count; used pages in random order."""
    common, more, ctx, chunk = _lengths(case)
    used = [-(-(c + n) // PAGE) for c, n in zip(ctx, chunk)]
    n_common, n_more, group = common // PAGE, more // PAGE, case.get("group", 1)
    n_groups = -(-len(ctx) // group) if n_more else 0
    own_pages = [u - n_common - n_more for u in used]
    n_pages = n_common + n_groups * n_more + sum(own_pages) + 3
    ids = np_rng.permutation(n_pages)
    table = np.zeros((len(ctx), max(used)), dtype=np.int32)
    at = n_common + n_groups * n_more
    for i, n in enumerate(own_pages):
        g = i // group
        table[i, :n_common] = ids[:n_common]
        table[i, n_common:n_common + n_more] = ids[n_common + g * n_more:n_common + (g + 1) * n_more]
        table[i, n_common + n_more:used[i]] = ids[at:at + n]
        at += n
    return torch.from_numpy(table), n_pages


def _frequencies(case):
    """Angle per position of each rotating pair (64 bits), and the factor on cosine and sine."""
    s, d = SCALINGS[case["scaling"]], case["rotary"]
    kind, factor = s["scaling"], s.get("factor", 1.0)
    i = np.arange(d // 2, dtype=np.float64)
    base = BASE * factor ** (d / (d - 2.0)) if kind == "base" and d > 2 else BASE
    f = base ** (-2.0 * i / d)
    if kind == "linear":
        return f / factor, 1.0
    if kind in ("turns", "index"):
        if kind == "turns":   # a frequency keeps its value from `high` turns over the original length on, is divided below `low`
            keep = (s["original_len"] * f / (2.0 * math.pi) - s["low"]) / (s["high"] - s["low"])
            amplitude = 1.0
        else:                 # the same between the indices of those frequencies, rounded outwards
            at = [d * math.log(s["original_len"] / (t * 2.0 * math.pi)) / (2.0 * math.log(BASE)) for t in (s["high"], s["low"])]
            first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), d - 1)
            keep = 1.0 - (i - first) / (last - first if last > first else 0.001)
            amplitude = 0.1 * math.log(factor) + 1.0
        keep = np.clip(keep, 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), amplitude
    return f, 1.0


_models = {}


def _model(hq, hkv, hd):
    """A server loads its model once: the operators take its head geometry from it."""
    import paper_2511_07423_b200 as syn
    from workloads.configs import ModelShape
    if (hq, hkv, hd) not in _models:
        shape = ModelShape("heads", 1, 128, hq, hkv, hd, 128, 128)

        def w(*size):
            return torch.zeros(*size, dtype=torch.bfloat16, device="cuda")

        glob = {"embed": w(128, 128), "lm_head": w(128, 128), "final_norm": w(128)}
        layer = {"wq": w(hq * hd, 128), "wk": w(hkv * hd, 128), "wv": w(hkv * hd, 128), "wo": w(128, hq * hd), "wg": w(128, 128),
                 "wu": w(128, 128), "wd": w(128, 128), "norm1": w(128), "norm2": w(128)}
        _models[hq, hkv, hd] = syn.Model(shape, glob, [layer])
    return _models[hq, hkv, hd]


def _projections(case, tokens, gen):
    """q, k, v as a projection leaves them: slices of one row per token, or arrays of their own."""
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    t = DTYPES[case["dtype"]]

    def normal(*size):
        return torch.empty(*size, dtype=t, device="cuda").normal_(0.0, 1.3, generator=gen)

    if case["fused"]:
        row = normal(tokens, hq + 2 * hkv, hd)
        return row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]
    return normal(tokens, hq, hd), normal(tokens, hkv, hd), normal(tokens, hkv, hd)


def _gains(case, gen):
    if not case["norm"]:
        return None, None
    return tuple(torch.empty(case["hd"], dtype=torch.float32, device="cuda").normal_(1.0, 0.1, generator=gen).to(torch.bfloat16) for _ in range(2))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    np_rng = np.random.default_rng(seed)
    st = {"case": case}
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    if own:
        import paper_2511_07423_b200 as syn
        st["syn"] = syn
    if case["op"] != "prefix":
        f, st["amplitude"] = _frequencies(case)
        st["freq"] = torch.from_numpy(f).cuda()
        if own:
            st["rope"] = syn.Rope(case["rotary"], BASE, case["layout"], **SCALINGS[case["scaling"]])
    if case["op"] == "rope":
        st["q"], st["k"], _ = _projections(case, case["tokens"], gen)
        st["q_gain"], st["k_gain"] = _gains(case, gen)
        far = case["far"]
        st["pos"] = torch.randint(max(0, far - far // 2), far, (case["tokens"],), generator=gen, device="cuda", dtype=torch.int32)
        if own:
            st["q_out"], st["k_out"] = torch.empty_like(st["q"].contiguous()), torch.empty_like(st["k"].contiguous())
        return st
    _, _, ctx, chunk = _lengths(case)
    tables, n_pages = _tables(case, np_rng)
    tokens = sum(chunk)
    offsets = torch.tensor([0] + list(np.cumsum(chunk)), dtype=torch.int32)
    pool_size = (n_pages, hkv, 2, PAGE, hd)
    if own:
        st["kv"] = syn.KVCache(_model(hq, hkv, hd), n_pages)
        st["pool"] = st["kv"].layer_view(0)
        st["plan"] = syn.Plan(st["kv"], torch.zeros(tokens, dtype=torch.int32), offsets, tables, torch.tensor(ctx, dtype=torch.int32),
                              share_prefix=case["op"] == "prefix")
    else:
        st["pool"] = torch.empty(pool_size, dtype=torch.float16, device="cuda")
    st["pool"].normal_(0.0, 1.0, generator=gen)
    # request and position of every token, for the plain form
    req = np.repeat(np.arange(len(ctx)), chunk)
    j = np.arange(tokens) - offsets.numpy()[req]
    pos = np.asarray(ctx)[req] + j
    st["req"], st["j"], st["pos"] = (torch.from_numpy(a.astype(np.int64)).cuda() for a in (req, j, pos))
    st["tables"] = tables.to(torch.int64).cuda()
    if case["op"] == "append":
        st["q"], st["k"], st["v"] = _projections(case, tokens, gen)
        st["q_gain"], st["k_gain"] = _gains(case, gen)
        if own and case["queries"]:
            st["q_out"] = torch.empty(tokens, hq * hd, dtype=torch.float16, device="cuda")
        return st
    st["q"] = torch.empty(tokens, hq * hd, dtype=torch.float16, device="cuda").normal_(0.0, 1.3, generator=gen)
    if own:
        st["out"] = torch.empty_like(st["q"])
    return st


# ------------------------------------------------------------------------------------------ one pass

def _norm_rotate(st, x, gain, pos):
    """[tokens, heads, hd] in 32 bits: the norm of each head, then the rotation (angles in 64 bits)."""
    case = st["case"]
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
    angle = pos.double()[:, None] * st["freq"]
    c, s = (st["amplitude"] * angle.cos()).float()[:, None], (st["amplitude"] * angle.sin()).float()[:, None]
    d = case["rotary"]
    turn, rest = x[..., :d], x[..., d:]
    if case["layout"] == "half":
        a, b = turn[..., :d // 2], turn[..., d // 2:]
        turn = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turn, rest], -1)


def _half(x):
    return x.clamp(-HALF_MAX, HALF_MAX).to(torch.float16)


def _plain_append(st):
    case = st["case"]
    page, row = st["tables"][st["req"], st["pos"] // PAGE], st["pos"] % PAGE
    st["pool"][page, :, 0, row] = _half(_norm_rotate(st, st["k"], st["k_gain"], st["pos"]))
    st["pool"][page, :, 1, row] = _half(st["v"].float())
    if not case["queries"]:
        return {"pool": st["pool"]}
    return {"pool": st["pool"], "q": _half(_norm_rotate(st, st["q"], st["q_gain"], st["pos"])).flatten(1)}


def _plain_attention(st):
    """Softmax over every request's own copy of its keys, padded to the longest request and the longest chunk."""
    case, pool, tables = st["case"], st["pool"], st["tables"]
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    g, b, n = hq // hkv, tables.shape[0], case["chunk_hi"]
    k, v = (pool[:, :, i][tables].permute(0, 2, 1, 3, 4).reshape(b, hkv, -1, hd).float() for i in range(2))
    q = torch.zeros(b, n, hkv, g, hd, device="cuda")
    q[st["req"], st["j"]] = st["q"].float().view(-1, hkv, g, hd)
    last = torch.zeros(b, n, dtype=torch.int64, device="cuda")
    last[st["req"], st["j"]] = st["pos"]
    s = q.permute(0, 2, 1, 3, 4).reshape(b, hkv, n * g, hd) @ k.transpose(-1, -2) / math.sqrt(hd)
    hidden = torch.arange(k.shape[2], device="cuda") > last.repeat_interleave(g, 1)[:, None, :, None]
    s.masked_fill_(hidden, -math.inf)
    p = s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = p @ v / p.sum(-1, keepdim=True)
    o = o.view(b, hkv, n, g, hd).permute(0, 2, 1, 3, 4)[st["req"], st["j"]]
    return o.reshape(-1, hq * hd).to(torch.float16)


def run(state):
    op = state["case"]["op"]
    if op == "rope":
        if own:
            return state["syn"].syn_op_qk_rope(state["rope"], state["q"], state["k"], state["pos"], state["q_gain"], state["k_gain"], EPS,
                                               state["q_out"], state["k_out"])
        return tuple(_norm_rotate(state, state[x], state[x + "_gain"], state["pos"]).to(state[x].dtype) for x in "qk")
    if op == "append":
        if own:
            q = state["plan"].append(0, state["k"], state["v"], state["rope"], state["k_gain"], state["q"] if state["case"]["queries"] else None,
                                     state["q_gain"], state.get("q_out"))
            return {"pool": state["pool"]} if q is None else {"pool": state["pool"], "q": q}
        return _plain_append(state)
    if own:
        return state["plan"].attention(0, state["q"], state["out"])
    return _plain_attention(state)


# ------------------------------------------------------------------------------------------ work and exact values

def work(case):
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    if case["op"] == "rope":
        values = case["tokens"] * (hq + hkv) * hd
        return {"bytes": 2 * values * DTYPES[case["dtype"]].itemsize, "flops": values * (3 + 4 * case["norm"])}
    common, more, ctx, chunk = _lengths(case)
    tokens = sum(chunk)
    if case["op"] == "append":
        q_heads = hq if case["queries"] else 0
        size = DTYPES[case["dtype"]].itemsize + 2   # read as the projection left it, written in half precision
        return {"bytes": tokens * (q_heads + 2 * hkv) * hd * size, "flops": tokens * (q_heads + hkv) * hd * (3 + 4 * case["norm"])}
    groups = -(-case["requests"] // case["group"])
    keys = common + groups * more + sum(c - common - more + n for c, n in zip(ctx, chunk))
    seen = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, chunk))
    return {"bytes": keys * hkv * hd * 4 + tokens * hq * hd * 4, "flops": 4 * hq * hd * seen}


def _exact_rotated(st, x, gain, pos):
    """The same from the definition: a rotating pair is a complex number, multiplied by e^(i angle)."""
    case = st["case"]
    x = x.double().clone()
    if gain is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * gain.double()
    f, amplitude = _frequencies(case)
    h = case["rotary"] // 2
    turn = torch.polar(torch.full_like(pos, amplitude, dtype=torch.float64)[:, None].expand(-1, h),
                       torch.outer(pos.double(), torch.from_numpy(f).to(pos.device)))[:, None]
    at = torch.arange(h, device=x.device)
    first, second = (at, at + h) if case["layout"] == "half" else (2 * at, 2 * at + 1)
    z = torch.complex(x[..., first], x[..., second]) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return x


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return tuple(_exact_rotated(st, st[x], st[x + "_gain"], st["pos"]) for x in "qk")
    if case["op"] == "append":
        pool = st["pool"].double()
        slot = st["tables"].gather(1, (st["pos"] // PAGE).clamp(max=st["tables"].shape[1] - 1)[None].expand(st["tables"].shape[0], -1))
        page = slot[st["req"], torch.arange(len(st["req"]), device="cuda")]
        new = torch.stack([_exact_rotated(st, st["k"], st["k_gain"], st["pos"]), st["v"].double()], 2)
        pool[page, :, :, st["pos"] % PAGE] = new.clamp(-HALF_MAX, HALF_MAX)
        if not case["queries"]:
            return {"pool": pool}
        return {"pool": pool, "q": _exact_rotated(st, st["q"], st["q_gain"], st["pos"]).clamp(-HALF_MAX, HALF_MAX).flatten(1)}
    _, _, ctx, chunk = _lengths(case)
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    out, at = [], 0
    for i, (c, n) in enumerate(zip(ctx, chunk)):   # one request after the other
        pages = st["pool"][st["tables"][i, :-(-(c + n) // PAGE)]].double()
        k, v = (pages[:, :, x].transpose(0, 1).reshape(hkv, -1, hd)[:, :c + n] for x in range(2))
        q = st["q"][at:at + n].double().view(n, hkv, hq // hkv, hd)
        s = torch.einsum("nhgd,hkd->hgnk", q, k) * hd ** -0.5
        s = torch.where(torch.ones(n, c + n, dtype=torch.bool, device="cuda").tril(c), s, -torch.inf)
        p = torch.exp(s - torch.logsumexp(s, -1, keepdim=True))
        out.append(torch.einsum("hgnk,hkd->nhgd", p, v).reshape(n, hq * hd))
        at += n
    return torch.cat(out)
