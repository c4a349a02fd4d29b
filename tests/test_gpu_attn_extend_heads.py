"""uniquan_attn_extend with many key/value heads: as many as leave two shares of each a place (256), and more.  Bars as in
extend_cases.check, on some of the heads."""
import numpy as np
import pytest

import extend_cases as X
import oracle.kv_cache as KV
from kv_cases import filled, on_device, rounded

pytestmark = pytest.mark.gpu


def some_heads(c, heads):
    """The cache's host copy with these key/value heads only."""
    s = KV.Cache(len(c.k), len(heads), c.d, c.P, c.fmt, c.group, c.table)
    s.k, s.v = c.k[:, heads], c.v[:, heads]
    if c.k_stat is not None:
        s.k_stat, s.v_stat = c.k_stat[:, heads], c.v_stat[:, heads]
    return s


@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("u8", 32), ("u4", None)])
@pytest.mark.parametrize("n_kv,grp,d,seqs", [
    (257, 1, 64, [(1, 700)]), (257, 2, 128, [(2, 900), (1, 300)]), (300, 1, 64, [(3, 600), (0, 400), (1, 1)]),
    (257, 1, 128, [(70, 300), (1, 520), (66, 66), (130, 290)]),     # more than 64 columns on average
    (257, 40, 128, [(4, 300), (1, 520), (2, 66), (1, 290)]),
    (256, 1, 64, [(1, 900), (2, 40)]), (171, 3, 128, [(2, 1500)]), (256, 9, 128, [(9, 700), (9, 300), (8, 8), (8, 1200)]),
])
def test_many_key_value_heads(fmt, group, n_kv, grp, d, seqs, monkeypatch):
    rs = np.random.default_rng(n_kv + grp)
    rows, lens = [s[0] for s in seqs], [s[1] for s in seqs]
    c = filled(rs, lens, n_kv, d, 64, fmt, group)
    m = on_device(c)
    T, H = sum(rows), n_kv * grp
    q = rounded(rs, T, H, d)
    heads = [0, 1, n_kv // 2, n_kv - 1]
    cols = np.concatenate([np.arange(g * grp, g * grp + min(grp, 3)) if grp < 4 else g * grp + np.arange(grp) for g in heads])
    real = X.call
    for kw in (dict(), dict(window=100, sinks=2)):
        O, l = real(c, m, q, X.starts(rows), lens, d ** -0.5, **kw)
        part = O.view(T, H, d)[:, cols].reshape(T, -1), l[:, cols]
        monkeypatch.setattr(X, "call", lambda *a, **k: part)
        X.check(some_heads(c, heads), None, q[:, cols], X.starts(rows), lens, d ** -0.5, **kw)
        monkeypatch.setattr(X, "call", real)
