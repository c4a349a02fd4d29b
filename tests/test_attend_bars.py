"""attend_bars on the host: a block of positions lost, doubled or exchanged breaks the bars in every format, and the
formula evaluated in fp32 with the weights in two bf16 terms keeps them."""
import numpy as np
import pytest

import oracle.kv_cache as KV
from attend_bars import BLOCK, LONG, bars, broken, long_rows, queries, store
from kv_cases import FORMS, attend_bounds, filled, rounded

F32 = np.float32


def weights(K, qh, scale):
    x = scale * (K @ qh.astype(np.float64))
    p = np.exp(x - x.max())
    return p / p.sum()


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shown", [True, False])
def test_a_block_gone_wrong_breaks_them(fmt, group, d, shown):
    rs = np.random.default_rng(80)
    lens = LONG
    c = long_rows(rs, lens, 1, d, 64, fmt, group, shown)
    q = queries(rs, len(lens), 2, d)
    scale = d ** -0.5
    want = bars(c, q, lens, scale)
    assert not any(b.any() for b in broken(want[0], c, q, lens, scale, want))
    for s, ln in enumerate(lens):
        if ln <= BLOCK:
            continue
        K, V = (x[0] for x in c.dense(s, ln))
        blocks = -(-ln // BLOCK)
        for h in range(2):
            p = weights(K, q[s, h], scale)
            for b in range(blocks):
                here = np.arange(b * BLOCK, min(ln, (b + 1) * BLOCK))
                there = here - BLOCK if b else here + BLOCK
                m = min(len(here), np.count_nonzero(there < ln))
                lost, twice, other = V.copy(), V.copy(), V.copy()
                lost[here] = 0
                twice[here] *= 2
                other[here[:m]], other[there[:m]] = V[there[:m]], V[here[:m]]
                gone = np.delete(np.arange(ln), here)  # with its part of the weights' sum
                for what, x in (("lost", p @ lost), ("twice", p @ twice), ("exchanged", p @ other),
                                ("left out", p[gone] @ V[gone] / p[gone].sum())):
                    got = want[0].copy()
                    got[s, h] = x
                    el, nrm = broken(got, c, q, lens, scale, want)
                    if len(here) < 32:  # a row's last few positions, in a part of a step
                        continue
                    assert (el if shown else nrm)[s, h], (what, s, h, b)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shown", [True, False])
def test_fp32_arithmetic_keeps_them(fmt, group, d, shown):
    rs = np.random.default_rng(81)
    lens = [2049, 300, 1]
    c = long_rows(rs, lens, 1, d, 64, fmt, group, shown)
    q = queries(rs, 3, 2, d)
    got = np.zeros(q.shape)
    for s, ln in enumerate(lens):
        K, V = (x[0].astype(F32) for x in c.dense(s, ln))
        for h in range(2):
            x = (F32(d ** -0.5) * (K @ q[s, h])).astype(F32)
            w = np.exp(x - x.max()).astype(F32)
            hi = (w.view(np.uint32) & 0xFFFF0000).view(F32)
            lo = ((w * F32(1 + 2.0 ** -17) - hi).astype(F32).view(np.uint32) & 0xFFFF0000).view(F32)
            o = ((hi @ V + lo @ V).astype(F32) / w.sum(dtype=F32)).astype(F32)
            got[s, h] = KV.from_bf16(KV.bf16(o))
    assert not any(b.any() for b in broken(got, c, q, lens, d ** -0.5))


def test_stored_as_one_by_one():
    """attend_bars.store writes what Cache.put writes."""
    for fmt, group in FORMS:
        a, b = (long_rows(np.random.default_rng(1), [40, 17], 3, 64, 16, fmt, group, False) for _ in range(2))
        rs = np.random.default_rng(2)
        for key in (True, False):
            x = rs.standard_normal((17, 3, 64)).astype(F32)
            store(a, key, 1, np.arange(17), x)
            for p in range(17):
                b.put(key, b.page(1, p), p % 16, x[p])
        for name in ("k", "v", "k_stat", "v_stat"):
            assert fmt == "bf16" and "stat" in name or np.array_equal(getattr(a, name), getattr(b, name))


@pytest.mark.parametrize("fmt,group", [f for f in FORMS if f[0] != "bf16"])
def test_the_wider_bars_let_a_block_go(fmt, group):
    """What kv_cases.attend_bounds, for codes, one large key channel and thousands of positions, does not see: a
    block's values lost.  These bars do."""
    rs = np.random.default_rng(6)
    c = filled(rs, [5000], 1, 128, 64, fmt, group)
    q = rounded(rs, 1, 4, 128)
    O, _, wide, _ = attend_bounds(c, q, [5000], 0.088)
    want = bars(c, q, [5000], 0.088)
    K, V = (x[0] for x in c.dense(0, 5000))
    V[1280:1280 + BLOCK] = 0
    got = np.stack([weights(K, q[0, h], 0.088) @ V for h in range(4)])[None]
    assert np.all(np.abs(got - O) <= wide)
    assert broken(got, c, q, [5000], 0.088, want)[1].all()
