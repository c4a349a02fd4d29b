"""How far a value comes back from its code, over fp32's range (oracle/kv_cache.py, which the device equals bit for
bit): half a scale, except for the smallest spreads (scale 0) and those near the largest fp32 number."""
import numpy as np
import pytest

import oracle.kv_cache as KV

F32 = np.float32


def groups(rs, e):
    """Groups of 32 whose spreads are about 2^e, around offsets of other sizes."""
    x = rs.uniform(-1, 1, (300, 32)) * 2.0 ** e
    off = rs.choice([0, 0, 1, -3, 100], (300, 1)) * 2.0 ** min(e, 118)
    return (x + off).astype(F32)


def back(x, fmt):
    c, sc, lo = KV.encode(x, fmt, 32)
    with np.errstate(all="ignore"):
        y = (lo + sc * c.astype(F32)).astype(F32).astype(np.float64)
        spread = (x.max(-1, keepdims=True) - lo).astype(F32)
    return y, sc.astype(np.float64), lo, spread


@pytest.mark.parametrize("fmt", ["u8", "u4"])
def test_within_half_a_scale(fmt):
    """Spreads from fp32's smallest numbers to below 2^127.  Three roundings of fp32 come on top: of x - lo, of the
    product with 1 / scale, of lo + scale code, each 2^-24 of the largest magnitude at most."""
    rs = np.random.default_rng(1)
    top = KV.TOP[fmt]
    for e in range(-140, 126):
        x = groups(rs, e)
        y, sc, lo, spread = back(x, fmt)
        assert np.isfinite(sc).all() and (spread < 2.0 ** 127).all()
        off = np.abs(y - x)
        some = sc[:, 0] > 0
        size = np.maximum(np.abs(x).max(-1, keepdims=True), np.abs(lo))
        assert np.all(off[some] <= 0.5 * sc[some] + 3 * 2.0 ** -24 * size[some] + 3 * 2.0 ** -150)
        # the spread is fl(max - lo): the exact one, which bounds `off`, is within 2^-24 / (1 - 2^-24) < 2^-23 of it
        assert np.all(off[~some] <= spread[~some].astype(np.float64) * (1 + 2.0 ** -23) + 2.0 ** -149)
        assert np.all(spread[~some] < top * 2.0 ** -126)
        if e < -130:
            assert not some.all()


@pytest.mark.parametrize("fmt", ["u8", "u4"])
def test_spreads_near_the_largest_number(fmt):
    """From 2^127 on: NaN as a whole, or each value within half a scale, or infinite."""
    rs = np.random.default_rng(2)
    x = np.stack([np.linspace(-3.0e38, hi, 32) for hi in rs.uniform(0, 0.5e38, 3000)]).astype(F32)
    y, sc, lo, spread = back(x, fmt)
    nan = np.isnan(sc[:, 0])
    assert np.array_equal(nan, ~np.isfinite(spread[:, 0])) and nan.any() and not nan.all()
    assert np.isnan(y[nan]).all()
    off = np.abs(y - x)[~nan]
    assert np.all((off <= 0.5 * sc[~nan] + 3 * 2.0 ** -24 * 3.5e38) | np.isposinf(y[~nan]))
