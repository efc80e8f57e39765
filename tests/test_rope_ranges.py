"""Descriptions of a rotation whose numbers leave their range are refused: an infinite base would leave all pairs but the first where
they are, an infinite angle or amplitude makes no numbers, one of zero makes zeros."""
import math

import pytest

import paper_2511_07423_b200 as syn


@pytest.mark.parametrize("args,kw", [
    ((128, 1e300), dict(scaling="base", factor=1e10)),                   # 1e300 * 1e10^(128 / 126)
    ((128, 1e-300), dict(scaling="base", factor=1e-10)),                 # zero
    ((128, 1e-310), {}),                                                 # f of the last pair 1e305, times 2^31
    ((128, 1e4), dict(scaling="linear", factor=1e-308)),
    ((64,), dict(amplitude=1e39)), ((64,), dict(amplitude=1e-46)),
])
def test_numbers_out_of_range_are_refused(args, kw):
    with pytest.raises(syn.SynError) as e:
        syn.Rope(*args, **kw)
    assert e.value.code == -1


@pytest.mark.parametrize("args,kw", [((128, 1e300), {}), ((64, 1e-200), {}), ((2, 1e300), dict(scaling="base", factor=1e10)),
                                     ((64,), dict(amplitude=1e38)), ((64,), dict(amplitude=2e-38))])
def test_far_but_within(args, kw):
    f, a = syn.Rope(*args, **kw).frequencies()
    d = args[0]
    base = args[1] if len(args) > 1 else 10000.0
    assert all(float(x) == pytest.approx(base ** (-2 * i / d), rel=1e-12) and math.isfinite(float(x) * 2 ** 31) for i, x in enumerate(f))
    assert a == kw.get("amplitude", 1.0)
