"""Pins of oracle/kv_cache.py on the host: the quantiser's guarantee, the row
orders, paging, and attention against a direct computation."""
import numpy as np
import pytest

import oracle.kv_cache as KV

F32 = np.float32


@pytest.mark.parametrize("fmt,group", [("u8", 32), ("u8", 128), ("u4", 32), ("u4", 128)])
def test_codes_come_back_within_half_a_scale(fmt, group):
    rs = np.random.default_rng(1)
    for f in (1.0, 1e-30, 1e30):
        x = (rs.standard_normal((50, 128)) * f + rs.standard_normal((50, 1)) * 3 * f).astype(F32)
        c, sc, lo = KV.encode(x, fmt, group)
        back = (lo[..., None].astype(np.float64) + sc[..., None].astype(np.float64) * c.reshape(50, -1, group)).reshape(50, 128)
        assert np.all(np.abs(back - x) <= np.repeat(sc, group, -1) * 0.5001)
        assert np.all(KV.bits(sc) & 0xFFFF == 0) and np.all(KV.bits(lo) & 0xFFFF == 0)


def test_edge_groups():
    x = np.zeros((5, 32), F32)
    x[1] = 2.5
    x[2, 3] = np.inf
    x[3, 3] = np.nan
    x[4, 0], x[4, 1] = -3e38, 3e38
    c, sc, lo = KV.encode(x, "u4", 32)
    assert np.all(c[:2] == 0) and sc[0, 0] == 0 and lo[0, 0] == 0 and sc[1, 0] == 0 and lo[1, 0] == 2.5
    assert np.isnan(sc[2:]).all() and np.isnan(lo[2:]).all() and np.all(c[2:] == 0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", ["u8", "u4"])
@pytest.mark.parametrize("key", [True, False])
def test_rows(d, fmt, key):
    assert sorted(KV.place(d, fmt, key)) == list(range(d))
    c = np.random.default_rng(2).integers(0, KV.TOP[fmt] + 1, (7, d)).astype(np.uint8)
    row = KV.pack(c, fmt, key)
    assert row.shape[-1] == (d if fmt == "u8" else d // 2)
    assert np.array_equal(KV.unpack(row, fmt, key), c)


def test_directed_rounding():
    x = np.array([1.0, 1.0000001, -1.0000001, -1e-40, 1e-40, 3.0e38, -3.0e38], F32)
    d = KV.down(x)
    assert np.all(d <= x) and np.all(KV.bits(d) & 0xFFFF == 0)
    assert d[0] == 1 and d[1] == 1 and d[2] == -1.0078125
    y = np.abs(x[:6])
    u = KV.up(y)
    assert np.all(u >= y) and np.all(KV.bits(u) & 0xFFFF == 0) and u[0] == 1 and u[1] == 1.0078125


def test_append_skips_padding_and_missing_pages():
    rs = np.random.default_rng(3)
    c = KV.Cache(4, 2, 64, 16, "bf16", 0, [[2, -1], [0, 7]])
    x = rs.standard_normal((6, 2, 64)).astype(F32)
    q = np.full((6, 2 * 64), 9, np.uint16)
    c.append(x, x, [3, 17, -1, 4, 20, 40], q=x, q_out=q, seq=[0, 0, 0, 1, 1, 1])
    held = [(p, r) for p in range(4) for r in range(16) if c.k[p, :, r].any()]
    assert held == [(0, 4), (2, 3)]
    assert np.all(q[[2, 5]] == 9) and not np.any(q[[0, 1, 3, 4]] == 9)


def test_attend_against_direct():
    rs = np.random.default_rng(4)
    c = KV.Cache(6, 2, 64, 16, "u8", 32, [[5, 1, 0], [2, -1, 3]])
    for s, n in ((0, 37), (1, 40)):
        for p in range(n):
            page = c.page(s, p)
            if page >= 0:
                for key in (True, False):
                    c.put(key, page, p % 16, rs.standard_normal((2, 64)).astype(F32))
    q = rs.standard_normal((2, 4, 64)).astype(F32)
    O, lse, _, _ = c.attend(q, [37, 40], 0.125)
    K, V = c.read([37, 40], 40)
    for s in range(2):
        ok = [p for p in range([37, 40][s]) if c.page(s, p) >= 0]
        assert len(ok) == (37 if s == 0 else 24)
        for h in range(4):
            x = 0.125 * K[h // 2, s, ok].astype(np.float64) @ q[s, h].astype(np.float64)
            p = np.exp(x)
            assert np.allclose(O[s, h], p @ V[h // 2, s, ok] / p.sum(), rtol=1e-6, atol=1e-7)
            assert abs(lse[s, h] - np.log2(p.sum())) < 1e-6
    assert np.all(c.attend(q, [0, 0], 1.0)[0] == 0) and np.all(np.isneginf(c.attend(q, [0, -3], 1.0)[1]))
