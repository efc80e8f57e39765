"""Rotation handles without a device: frequencies of every scaling against the formulas, and refusals."""
import math

import numpy as np
import pytest
import torch

import paper_2511_07423_b200 as syn


def formula(d, base, scaling, factor=1.0, original_len=0.0, low=0.0, high=0.0):
    i = np.arange(d // 2, dtype=np.float64)
    f = base ** (-2 * i / d)
    if scaling == "none":
        return f
    if scaling == "linear":
        return f / factor
    if scaling == "base":
        return (base * factor ** (d / (d - 2))) ** (-2 * i / d) if d > 2 else f
    if scaling == "turns":
        keep = (original_len * f / (2 * math.pi) - low) / (high - low)
    else:
        a, b = (d * math.log(original_len / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (high, low))
        first, last = max(math.floor(a), 0), min(math.ceil(b), d - 1)
        keep = 1 - (i - first) / (last - first if last > first else 0.001)
    keep = np.clip(keep, 0, 1)
    return f * keep + f / factor * (1 - keep)


CASES = [
    (128, 10000.0, dict(scaling="none")),
    (2, 500000.0, dict(scaling="none")),
    (2, 500000.0, dict(scaling="base", factor=4.0)),
    (64, 10000.0, dict(scaling="linear", factor=4.0)),
    (80, 10000.0, dict(scaling="base", factor=8.0)),
    (128, 500000.0, dict(scaling="turns", factor=8.0, original_len=8192.0, low=1.0, high=4.0)),
    (256, 1e6, dict(scaling="index", factor=16.0, original_len=4096.0, low=1.0, high=32.0)),
    (54, 10000.0, dict(scaling="index", factor=2.5, original_len=2048.0, low=1.0, high=32.0)),
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,base,kw", CASES)
def test_frequencies(d, base, kw, layout):
    f, a = syn.Rope(d, base, layout, **kw).frequencies()
    # a few operations in 64 bits on each side, a power among them: relative 1e-14
    np.testing.assert_allclose(f.numpy(), formula(d, base, **kw), rtol=1e-14, atol=0)
    assert a == pytest.approx(0.1 * math.log(kw["factor"]) + 1 if kw["scaling"] == "index" else 1.0, rel=1e-15)


def test_a_given_amplitude_is_taken():
    assert syn.Rope(64, amplitude=1.25).frequencies()[1] == 1.25
    assert syn.Rope(64, 1e4, scaling="index", factor=4.0, original_len=100.0, low=1.0, high=2.0, amplitude=0.5).frequencies()[1] == 0.5


@pytest.mark.parametrize("args,kw", [
    ((0,), {}), ((3,), {}), ((258,), {}), ((64, 0.0), {}), ((64, -1.0), {}), ((64, math.nan), {}), ((64, math.inf), {}),
    ((64, 1e4, "quarters"), {}), ((64,), dict(scaling="log")), ((64,), dict(scaling="linear", factor=0.0)),
    ((64,), dict(amplitude=-1.0)), ((64,), dict(amplitude=math.nan)), ((-2,), {}),
    ((64,), dict(scaling="turns", factor=2.0, original_len=0.0, low=1.0, high=4.0)),
    ((64,), dict(scaling="turns", factor=2.0, original_len=10.0, low=4.0, high=4.0)),
    ((64,), dict(scaling="index", factor=2.0, original_len=10.0, low=0.0, high=4.0)),
    ((64, 1.0), dict(scaling="index", factor=2.0, original_len=10.0, low=1.0, high=4.0)),
])
def test_refusals(args, kw):
    with pytest.raises(syn.SynError) as e:
        syn.Rope(*args, **kw)
    assert e.value.code == -1


def test_c_entries_refuse_null_pointers():
    import ctypes as C
    lib = syn.load_library()
    out = C.c_void_p()
    assert lib.syn_rope_create(None, C.byref(out)) == -1
    assert lib.syn_rope_freqs(None, None, None) == -1
    assert lib.syn_kv_layer(None, C.c_uint32(0), C.byref(out), C.byref(C.c_int64())) == -1
    assert lib.syn_op_qk_rope(None, None, None, None, 1, 64, 1e-5, 0, 0, None) == -1
    assert lib.syn_op_kv_append(None, None, None, 0, None, None, None, None, 0, None) == -1



def test_the_c_entry_checks_shapes_before_it_touches_the_device():
    """Made-up addresses: a refused call reads none of them."""
    import ctypes as C
    from paper_2511_07423_b200 import binding
    lib = syn.load_library()
    rope = syn.Rope(64)

    def call(x=1 << 20, y=1 << 30, gain=None, xs=256, ys=256, heads=4, T=3, hd=64, eps=1e-5, it=0, ot=0, pos=1 << 12, r=rope):
        h = binding._Heads(x, y, gain, xs, ys, heads)
        return lib.syn_op_qk_rope(r._h if r else None, C.addressof(h), None, pos, T, hd, eps, it, ot, None)

    assert call(T=-1) == -1
    assert call(hd=60) == -1 and call(hd=264) == -1 and call(hd=0) == -1
    assert call(hd=32) == -1            # narrower than the rotation
    assert call(heads=0) == -1
    assert call(xs=255) == -1 and call(ys=255) == -1
    assert call(x=None) == -1 and call(y=None) == -1 and call(pos=None) == -1
    assert call(x=(1 << 20) + 1) == -1 and call(y=(1 << 30) + 1) == -1 and call(gain=(1 << 12) + 1) == -1
    assert call(pos=(1 << 12) + 2) == -1
    assert call(it=3) == -1 and call(it=-1) == -1 and call(it=1, ot=0) == -1 and call(it=0, ot=2) == -1
    assert call(eps=-1.0) == -1 and call(eps=math.nan) == -1
    assert call(y=1 << 20, ys=512) == -1                       # in place with another stride
    assert call(y=1 << 20, it=2, ot=1) == -1                   # in place with another size
    assert call(T=0) == 0                                      # nothing to do, nothing launched
