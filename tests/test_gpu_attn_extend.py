"""uniquan_attn_extend against oracle/kv_cache.py in 64 bits; bars in extend_cases.check."""
import numpy as np
import pytest
import torch

import extend_cases as X
import oracle.kv_cache as KV
from kv_cases import FORMS, dev, filled, on_device, rounded, tables
from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu
F32 = np.float32

SEQS = [(1, 1), (3, 3), (5, 40), (17, 17), (0, 9), (7, 33), (2, 65), (0, 0), (12, 130), (1, 64)]


def case(seqs, n_kv, grp, d, P, fmt, group, seed=0, **kw):
    rs = np.random.default_rng(seed + 10 * n_kv + grp)
    rows, lens = [s[0] for s in seqs], [s[1] for s in seqs]
    c = filled(rs, lens, n_kv, d, P, fmt, group, **kw)
    return rs, c, on_device(c), rounded(rs, sum(rows), n_kv * grp, d), X.starts(rows), lens


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_kv,grp,P", [(2, 1, 16), (1, 8, 64), (3, 3, 32), (1, 21, 128)])
def test_rows_behind_what_is_cached(fmt, group, d, n_kv, grp, P):
    """Each row sees what lies before it: lengths around tiles and pages, sequences without rows."""
    rs, c, m, q, start, lens = case(SEQS, n_kv, grp, d, P, fmt, group)
    X.check(c, m, q, start, lens, d ** -0.5)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d,n_kv,grp", [(64, 2, 4), (128, 1, 1), (128, 2, 5)])
def test_trees(fmt, group, d, n_kv, grp):
    """Drafts see their ancestors; masks drawn bit by bit; rows whose mask is empty, with and without a history."""
    seqs = [(4, 4), (9, 30), (33, 50), (1, 1), (20, 147), (3, 32), (0, 5)]
    rs, c, m, q, start, lens = case(seqs, n_kv, grp, d, 16, fmt, group)
    paths = sum((X.tree(rs, r)[1] for r, _ in seqs), [])
    X.check(c, m, q, start, lens, d ** -0.5, mask=paths, what="paths")
    drawn = [int(rs.integers(0, 1 << 62)) for _ in paths]
    drawn[0] = drawn[5] = 0
    drawn[1] = (1 << 64) - 1                        # bits past the rows
    X.check(c, m, q, start, lens, d ** -0.5, mask=drawn, what="drawn")


@pytest.mark.parametrize("words", [2, 3, 64])
def test_large_trees(words):
    seqs = [(100, 131), (64, 64), (128, 300), (65, 70)]
    rs, c, m, q, start, lens = case(seqs, 2, 2, 64, 32, "bf16", 0)
    paths = sum((X.tree(rs, r, back=60)[1] for r, _ in seqs), [])
    X.check(c, m, q, start, lens, 0.125, mask=paths, words=words)
    drawn = [int.from_bytes(rs.bytes(16), "little") for _ in paths]
    X.check(c, m, q, start, lens, 0.125, mask=drawn, words=words)


def test_a_mask_word_too_few_hides_the_rest():
    seqs = [(70, 80)]
    rs, c, m, q, start, lens = case(seqs, 1, 1, 64, 16, "u8", 32)
    full = [(1 << 128) - 1] * 70
    O, l = X.call(c, m, q, start, lens, 0.125, mask=[(1 << 64) - 1] * 70, words=1)
    X.check(c, m, q, start, lens, 0.125, mask=[(1 << 64) - 1] * 70, words=1)
    O2, l2 = X.call(c, m, q, start, lens, 0.125, mask=full, words=2)
    assert not torch.equal(l, l2)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (31, 4), (32, 0), (64, 40), (100, 33), (1000, 3), (1 << 30, 0),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("d,n_kv,grp", [(64, 2, 3), (128, 1, 9)])
def test_windows(fmt, group, window, sinks, d, n_kv, grp):
    seqs = [(1, 200), (9, 140), (40, 40), (3, 300), (0, 3), (1, 1)]
    rs, c, m, q, start, lens = case(seqs, n_kv, grp, d, 16, fmt, group)
    X.check(c, m, q, start, lens, 0.125, window=window, sinks=sinks, what="rows")
    at = [ln - r + j for r, ln in seqs for j in range(r)]
    O, l = X.call(c, m, q, start, lens, 0.125, window=window, sinks=sinks)
    O2, l2 = X.call(c, m, q, start, lens, 0.125, window=window, sinks=sinks, pos=at)
    assert torch.equal(O, O2) and torch.equal(l, l2)
    depth, path = [], []
    for r, ln in seqs:
        a, b = X.tree(rs, r)
        depth += [ln - r + x for x in a]
        path += b
    X.check(c, m, q, start, lens, 0.125, window=window, sinks=sinks, mask=path, pos=depth, what="trees")
    far = rs.integers(-50, 400, len(path))          # positions of other axes
    far[0], far[1] = 2 ** 31 - 1, -2 ** 31
    X.check(c, m, q, start, lens, 0.125, window=window, sinks=sinks, mask=path, pos=far, what="trees, positions apart")
    X.check(c, m, q, start, lens, 0.125, window=window, sinks=sinks, pos=far, what="rows, positions apart")


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d,n_kv,grp,rows", [(128, 1, 1, 1), (128, 1, 8, 2), (64, 2, 8, 5), (128, 2, 4, 30)])
def test_long_sequences_cut_into_shares(fmt, group, d, n_kv, grp, rows):
    seqs = [(rows, 5003), (rows, 40), (0, 700), (rows, 1500), (rows, rows)]
    rs, c, m, q, start, lens = case(seqs, n_kv, grp, d, 64, fmt, group)
    assert uq.uniquan_attn_extend_ws(4 * rows, 5, n_kv * grp, n_kv, d, m["table"].shape[1], 64) > 0
    X.check(c, m, q, start, lens, d ** -0.5)
    X.check(c, m, q, start, lens, d ** -0.5, window=3000, sinks=50)
    path = sum((X.tree(rs, r)[1] for r, _ in seqs), [])
    X.check(c, m, q, start, lens, d ** -0.5, mask=path)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_many_tiles(fmt, group, d):
    """A prompt's part of many rows; with pages of 16 that lie apart, holes among them."""
    rs, c, m, q, start, lens = case([(300, 420), (211, 211)], 2, 8, d, 16, fmt, group)
    X.check(c, m, q, start, lens, 0.125)
    c.table[0, 3] = c.table[0, 20] = c.table[1, 0] = -1
    X.check(c, on_device(c), q, start, lens, 0.125, what="holes")


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("n_kv,grp,rows", [(2, 4, (300, 1, 16, 17, 1, 0, 4, 5)), (1, 1, (1, 16, 17, 64, 65, 600, 0, 128)),
                                           (3, 8, (1, 2, 3, 8, 9, 150))])
def test_a_prompt_beside_single_tokens(fmt, group, n_kv, grp, rows):
    """Sequences of many and of few rows in one call (more than 64 columns on average; up to 16, or of codes in groups of
    32 up to 64, have tiles of their own), lengths of which some are cut into shares."""
    lens = [2500, 1999, 700, 33, 1, 40, 900, 1300][:len(rows)]
    seqs = [(r, max(r, ln)) for r, ln in zip(rows, lens)]
    assert -(-sum(rows) // len(rows)) * grp > 64
    rs, c, m, q, start, lens = case(seqs, n_kv, grp, 128, 32, fmt, group)
    X.check(c, m, q, start, lens, 0.09, what="rows")
    X.check(c, m, q, start, lens, 0.09, window=300, sinks=3, what="window")
    path = sum((X.tree(rs, r, back=40)[1] for r, _ in seqs), [])
    X.check(c, m, q, start, lens, 0.09, mask=path, words=10, what="trees")


def test_many_sequences():
    """More sequences than lanes, in runs of several a lane."""
    rs = np.random.default_rng(5)
    for n in (63, 64, 65, 200, 1000):
        seqs = [(int(rs.integers(0, 4)), int(rs.integers(4, 60))) for _ in range(n)]
        rs2, c, m, q, start, lens = case(seqs, 1, 2, 64, 16, "u4", 32, seed=n)
        X.check(c, m, q, start, lens, 0.125, what=f"{n} sequences")


@pytest.mark.parametrize("fmt,group", FORMS)
def test_pages_that_are_none_and_lengths_out_of_range(fmt, group):
    rs = np.random.default_rng(7)
    lens = [100, 90, 64, 33, 80, 70]
    t, n_pages = tables(rs, lens, 16, max_pages=7)
    t[0, 2] = t[1, 5] = -1
    t[1, 0] = n_pages
    t[2, :] = -1
    t[4, 1] = 2 ** 31 - 1
    t[4, 3] = -2 ** 31
    c = filled(rs, lens, 2, 64, 16, fmt, group, table=(t, n_pages))
    m = on_device(c)
    rows = [5, 8, 3, 6, 1, 4]
    q = rounded(rs, sum(rows), 4, 64)
    start = X.starts(rows)
    X.check(c, m, q, start, lens, 0.125, what="holes")
    X.check(c, m, q, start, lens, 0.125, window=20, sinks=2, what="holes, window")
    for other in ([5, 7, 0, -3, 1, 3], [0, 0, 0, 0, 0, 0], [-2 ** 31] * 6, [1000, 2 ** 31 - 1, 112, 113, 200, 120]):
        # fewer places than rows, none, more than the table holds (what lies there is poison)
        if max(other) > 100:
            other = [min(x, 10 ** 6) for x in other]
            full, n2 = tables(rs, [112] * 6, 16)
            c2 = filled(rs, [112] * 6, 2, 64, 16, fmt, group, table=(full, n2))
            X.check(c2, on_device(c2), q, start, other, 0.125, what=f"lengths {other}")
        else:
            X.check(c, m, q, start, other, 0.125, what=f"lengths {other}")


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d,grp", [(64, 1), (64, 6), (128, 2), (128, 5)])
def test_what_is_not_seen_may_be_anything(fmt, group, d, grp):
    """NaN and infinities in drafts of other branches, behind a window and behind a row's own place, in keys, values,
    scales and offsets: rows that see them may come out as they like, the others as without."""
    rs = np.random.default_rng(grp)
    m_rows, ln, P = 12, 60, 16
    c = filled(rs, [ln], 2, d, P, fmt, group)
    q = rounded(rs, m_rows, 2 * grp, d)
    start = X.starts([m_rows])
    base = ln - m_rows
    depth, path = X.tree(rs, m_rows)
    for at, kw in ((base + 4, dict(mask=path)), (base + 5, dict()), (20, dict(window=30, sinks=3)),
                   (base - 10, dict(window=15, sinks=1, mask=path, pos=[base + x for x in depth]))):
        page = c.page(0, at)
        saved = [None if a is None else a.copy() for a in (c.k, c.v, c.k_stat, c.v_stat)]
        good = X.call(c, on_device(c), q, start, [ln], d ** -0.5, **kw)
        clean = c.attend_rows(q, start, [ln], d ** -0.5, **kw)
        for bits in (0x7FC0, 0x7F80, 0xFF80):
            for a, st in ((c.k, c.k_stat), (c.v, c.v_stat)):
                if st is None:
                    a[page, :, at % P] = bits
                    a[page, :, at % P, 1::3] = 0x3F80
                else:
                    st[page, :, :, at % P] = bits
            bad = X.call(c, on_device(c), q, start, [ln], d ** -0.5, **kw)
            for a, s in zip((c.k, c.v, c.k_stat, c.v_stat), saved):
                if a is not None:
                    a[...] = s
            P_of = kw.get("pos", [base + j for j in range(m_rows)])
            for j in range(m_rows):
                near = not kw.get("window") or at < kw["sinks"] or at > P_of[j] - kw["window"]
                sees = near if at < base else (path[j] >> (at - base) & 1 if "mask" in kw else at <= base + j)
                if not sees:
                    assert torch.equal(good[0][j], bad[0][j]) and torch.equal(good[1][j], bad[1][j]), (at, kw, j, hex(bits))
        assert clean[4].min() >= 0


@pytest.mark.parametrize("d", [64, 128])
def test_infinite_values_that_are_seen(d):
    """An infinite value comes out infinite in its channel, of every row that sees it, the other channels finite."""
    rs = np.random.default_rng(d)
    c = filled(rs, [50], 1, d, 16, "bf16", 0)
    at, ch = 45, 5
    c.v[c.page(0, at), 0, at % 16, ch] = 0x7F80
    for grp, rows in ((1, 10), (4, 10)):
        q = rounded(rs, rows, grp, d)
        O, l = X.call(c, on_device(c), q, X.starts([rows]), [50], d ** -0.5)
        o = O.float().cpu().numpy().reshape(rows, grp, d)
        sees = np.arange(rows) + 40 >= at
        assert np.all(np.isposinf(o[sees][..., ch])) and np.all(np.isfinite(o[~sees]))
        assert np.all(np.isfinite(np.delete(o, ch, -1)))


@pytest.mark.parametrize("d", [64, 128])
def test_largest_values_of_a_bf16_cache(d):
    rs = np.random.default_rng(1)
    c = filled(rs, [600], 1, d, 16, "bf16", 0)
    c.v[...] = np.where(c.v == 0x7FC1, c.v, 0x7F7F)  # the largest finite number
    q = rounded(rs, 40, 2, d)
    O, _ = X.call(c, on_device(c), q, X.starts([40]), [600], 0.125)
    assert np.all(O.float().cpu().numpy() == np.float32(KV.from_bf16(np.uint16(0x7F7F))))


def test_rows_behind_the_last_sequence_and_before_the_first_stay():
    rs, c, m, q, start, lens = case([(3, 20), (4, 40)], 2, 2, 64, 16, "u8", None)
    q = rounded(rs, 12, 4, 64)
    X.check(c, m, q, start + 2, lens, 0.125)        # rows 2 .. 8 of 12
    X.check(c, m, q, start, lens, 0.125, lse=False)


def test_row_starts_out_of_range_are_not_followed():
    """Starts that a caller should not give: nothing outside the T rows is read or written."""
    rs, c, m, q, start, lens = case([(3, 20), (4, 40)], 1, 2, 64, 16, "bf16", 0)
    for bad in ([0, 3, 2], [-5, 3, 7], [3, 1, 0], [0, 2 ** 31 - 1, -2 ** 31], [0, 100, 200], [6, 6, 9]):
        O, l = X.call(c, m, q, np.array(bad, np.int32), lens, 0.125)
        assert O.shape == (7, 128)


@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("u4", 32)])
@pytest.mark.parametrize("scale", [-0.125, 0.0, 3.0])
def test_scales(fmt, group, scale):
    for d, grp in ((64, 2), (128, 9)):
        rs, c, m, q, start, lens = case(SEQS, 2, grp, d, 16, fmt, group)
        X.check(c, m, q, start, lens, scale)
        X.check(c, m, q, start, lens, scale, window=9, sinks=2)


@pytest.mark.parametrize("fmt,group", [("bf16", 0), ("u8", 32)])
def test_rows_apart(fmt, group):
    """Q and O as column slices of wider tensors; what lies beside O stays."""
    rs, c, m, q, start, lens = case(SEQS, 2, 3, 64, 16, fmt, group)
    T, H, d = q.shape
    O, l = X.call(c, m, q, start, lens, 0.125)
    wide = torch.full((T, H * d + 24), 5.0, device="cuda", dtype=torch.bfloat16)
    qw = torch.zeros(T, H * d + 40, device="cuda", dtype=torch.bfloat16)
    qw[:, 8:8 + H * d] = dev(q.reshape(T, -1)).bfloat16()
    l2 = torch.empty_like(l)
    uq.uniquan_attn_extend(T, len(lens), H, 2, d, qw[:, 8:8 + H * d], dev(start), dev(np.asarray(lens, np.int32)), scale=0.125,
                           O=wide[:, 4:4 + H * d], row_lse=l2, ws=X.workspace(T, len(lens), H, 2, d, m), **m)
    assert torch.equal(wide[:, 4:4 + H * d], O) and torch.equal(l, l2)
    assert (wide[:, :4] == 5).all() and (wide[:, 4 + H * d:] == 5).all()


def test_one_row_as_the_single_token_call():
    """One row per sequence sees what uniquan_attn_decode's does: both within their bars of 64 bits, and here equal to
    the sum of the two (2^-14 of the values' size each and half a step of bf16 each)."""
    rs, c, m, q, start, lens = case([(1, x) for x in (1, 30, 500, 77, 1024)], 2, 4, 128, 32, "u8", 128)
    O, l = X.check(c, m, q, start, lens, 0.09)
    O2, l2 = torch.empty_like(O), torch.empty_like(l)
    need = uq.uniquan_attn_decode_ws(5, 8, 2, 128, m["table"].shape[1], 32)
    uq.uniquan_attn_decode(5, 8, 2, 128, dev(q.reshape(5, -1)).bfloat16(), dev(np.asarray(lens, np.int32)), scale=0.09, O=O2,
                           row_lse=l2, ws=torch.empty(max(1, need), device="cuda"), **m)
    absv = torch.from_numpy(c.attend_rows(q, start, lens, 0.09)[2]).cuda()
    bar = (2.0 ** -13 + 2.0 ** -10) * absv.repeat_interleave(128, 1) + 2.0 ** -7 * O.float().abs()
    assert ((O.float() - O2.float()).abs() <= bar).all()


def test_same_results_every_time_and_on_another_stream():
    rs, c, m, q, start, lens = case([(40, 3000), (7, 900)], 2, 4, 128, 64, "u4", 32)
    want = X.call(c, m, q, start, lens, 0.09)
    side = torch.cuda.Stream()
    for _ in range(3):
        got = X.call(c, m, q, start, lens, 0.09)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = X.call(c, m, q, start, lens, 0.09)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_calls_at_once_with_a_workspace_each():
    rs, c, m, q, start, lens = case([(6, 3000), (7, 900)], 2, 4, 64, 64, "bf16", 0)
    T, H, d = q.shape
    q2 = rounded(rs, T, H, d)
    want = [X.call(c, m, x, start, lens, 0.125)[0] for x in (q, q2)]
    outs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    args = (dev(start), dev(np.asarray(lens, np.int32)))
    ops = [(dev(x.reshape(T, -1)).bfloat16(), torch.empty(T, H * d, device="cuda", dtype=torch.bfloat16),
            X.workspace(T, 2, H, 2, d, m)) for x in (q, q2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for (x, O, ws), st in zip(ops, streams):
            uq.uniquan_attn_extend(T, 2, H, 2, d, x, *args, scale=0.125, O=O, ws=ws, stream=st, **m)
    torch.cuda.synchronize()
    assert all(torch.equal(o[1], w) for o, w in zip(ops, want))


def test_captured_and_replayed_as_lengths_grow():
    rs = np.random.default_rng(3)
    lens0, rows = [500, 20, 130], [4, 0, 6]
    c = filled(rs, [600, 120, 230], 2, 64, 16, "u8", 32)
    m = on_device(c)
    T = 12
    q = rounded(rs, T, 4, 64)
    Q, start, lens = dev(q.reshape(T, -1)).bfloat16(), dev(X.starts(rows)), dev(np.asarray(lens0, np.int32))
    O, l = torch.zeros(T, 256, device="cuda", dtype=torch.bfloat16), torch.zeros(T, 4, device="cuda")
    ws = X.workspace(T, 3, 4, 2, 64, m)
    run = lambda: uq.uniquan_attn_extend(T, 3, 4, 2, 64, Q, start, lens, scale=0.125, O=O, row_lse=l, ws=ws,  # noqa: E731
                                         window=90, sinks=4, **m)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(4):
        lens += 20
        if i == 2:
            start.copy_(dev(X.starts([1, 5, 2])))
        O.fill_(7.0)
        l.fill_(7.0)
        ws.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        want = X.call(c, m, q, start.cpu().numpy(), lens.cpu().numpy(), 0.125, window=90, sinks=4)
        assert torch.equal(O, want[0]) and torch.equal(l, want[1]), f"replay {i}"


def test_offsets_past_32_bits():
    """A sequence on the last pages of a cache of more than 2^32 bytes."""
    P, d, n_kv, need = 64, 128, 8, 5
    n_pages = (1 << 32) // (n_kv * P * d * 2) + 40
    rs = np.random.default_rng(0)
    small = filled(rs, [300], n_kv, d, P, "bf16", 0)
    k, v = (torch.zeros(n_pages, n_kv, P, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    t = small.table[0, :need]
    last = np.arange(n_pages - need, n_pages)
    for a, b in zip(t, last):
        k[b], v[b] = dev(small.k[a]), dev(small.v[a])
    q = rounded(rs, 6, 16, d)
    want = X.call(small, on_device(small), q, [0, 6], [300], 0.09)
    m = dict(table=dev(last[None].astype(np.int32)), k_cache=k, v_cache=v, k_stat=None, v_stat=None, fmt=uq.KV_BF16, group=0,
             page_len=P)
    got = X.call(small, m, q, [0, 6], [300], 0.09)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
