"""uniquan_attn_extend over thousands of sequences: each finds its rows among all, and the time is theirs, not their
square.  Bars as in extend_cases.check; pages are shared, so that a large batch takes little memory."""
import numpy as np
import pytest
import torch

import extend_cases as X
from kv_cases import dev, filled, on_device, rounded
from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu


def shared(rs, n, mp, n_kv, d, P, pool, fmt, group):
    """A cache whose n sequences have mp pages each, drawn from a pool of full ones."""
    lens = [P * pool]
    c = filled(rs, lens, n_kv, d, P, fmt, group)
    c.table = rs.choice(c.table[0], (n, mp))
    return c


@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("u8", 32), ("u4", None)])
@pytest.mark.parametrize("d,n_kv,grp,n,most", [(64, 1, 1, 2500, 3), (128, 2, 4, 1100, 20), (128, 1, 30, 1030, 9),
                                               (64, 3, 2, 700, 40), (128, 1, 8, 600, 33)])
def test_against_the_oracle(fmt, group, d, n_kv, grp, n, most):
    """Sequences of drawn numbers of rows, many of none, behind rows of padding; some of hundreds of columns."""
    rs = np.random.default_rng(n)
    c = shared(rs, n, 3, n_kv, d, 16, 40, fmt, group)
    rows = np.where(rs.random(n) < 0.4, 0, rs.integers(0, most, n))
    rows[rs.integers(0, n, 3)] = 130
    rows[-1] = 1
    lens = rs.integers(0, 49, n)
    start = X.starts(rows) + 5
    q = rounded(rs, int(start[-1]) + 3, n_kv * grp, d)
    X.check(c, on_device(c), q, start, lens, d ** -0.5)


@pytest.mark.parametrize("rows,len_max", [(2, 900), (90, 60)])
def test_as_in_batches_of_ten_thousand(rows, len_max):
    """40000 sequences as they come out in four calls: the rows of each in the same tiles."""
    rs = np.random.default_rng(rows)
    n, n_kv, grp, d, P, part = 40000, 1, 1, 64 if rows < 50 else 128, 64, 10000
    c = shared(rs, n, 15, n_kv, d, P, 60, "bf16", 0)
    m = on_device(c)
    r = rs.integers(0, 2 * rows, n)
    start, lens = X.starts(r), dev(rs.integers(0, len_max, n).astype(np.int32))
    T = int(start[-1])
    g = torch.Generator(device="cuda").manual_seed(1)
    Q = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    want, got = torch.full_like(Q, 7.0), torch.full_like(Q, 7.0)
    table = m.pop("table")
    assert uq.uniquan_attn_extend_ws(T, n, 1, 1, d, table.shape[1], P) == 0
    uq.uniquan_attn_extend(T, n, 1, 1, d, Q, dev(start), lens, table, scale=0.1, O=got, **m)
    for a in range(0, n, part):
        s = start[a:a + part + 1]
        lo, hi = int(s[0]), int(s[-1])
        uq.uniquan_attn_extend(hi - lo, part, 1, 1, d, Q[lo:hi], dev(s - s[0]), lens[a:a + part], table[a:a + part], scale=0.1,
                               O=want[lo:hi], ws=X.workspace(hi - lo, part, 1, 1, d, dict(m, table=table[a:a + part])), **m)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_the_largest_number_of_sequences():
    """2^20 of one row: a search among them, not a sum over them, for each."""
    n, d, P = 1 << 20, 64, 16
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(100, 1, P, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(0, 100, (n, 1), generator=g, device="cuda", dtype=torch.int32)
    lens = torch.ones(n, dtype=torch.int32, device="cuda")
    start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    Q = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    O = torch.empty_like(Q)
    uq.uniquan_attn_extend(n, n, 1, 1, d, Q, start, lens, table, k, v, 0.1, O, page_len=P)
    torch.cuda.synchronize()
    assert torch.equal(O, v[table[:, 0].long(), 0, 0])


def test_few_rows_among_many_sequences():
    """Five rows in 20000 sequences, long ones that are cut among them."""
    rs = np.random.default_rng(9)
    n = 20000
    c = shared(rs, n, 40, 1, 128, 64, 50, "u8", 32)
    rows = np.zeros(n, int)
    rows[[0, 77, 12345, 19999]] = [1, 2, 1, 1]
    lens = rs.integers(0, 2560, n)
    lens[[0, 12345]] = 2560
    q = rounded(rs, 5, 2, 128)
    m = on_device(c)
    assert uq.uniquan_attn_extend_ws(5, n, 2, 1, 128, 40, 64) > 0
    X.check(c, m, q, X.starts(rows), lens, 0.09)
