"""Shared by the tests of uniquan_attn_extend: a call on device copies, and its bars against oracle.kv_cache in 64 bits."""
import numpy as np
import torch

from kv_cases import WIDE, dev
from paper_2506_03781_amd import uniquan as uq


def starts(rows):
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)


def words_of(mask, words):
    """Python integers as [T, words] 64-bit words on the device."""
    a = np.array([[(m >> (64 * w)) & (2 ** 64 - 1) for w in range(words)] for m in mask], np.uint64)
    return dev(a.view(np.int64).reshape(len(mask), words))


def workspace(T, n, H, n_kv, d, m, fill=float("nan")):
    need = uq.uniquan_attn_extend_ws(T, n, H, n_kv, d, m["table"].shape[1], m["page_len"])
    return torch.full((max(1, need),), fill, device="cuda")


def call(c, m, q, row_start, lens, scale, mask=None, words=1, pos=None, window=0, sinks=0, lse=True):
    T, H, d = q.shape
    n = len(lens)
    O = torch.full((T, H * d), 7.0, device="cuda", dtype=torch.bfloat16)
    l = torch.full((T, H), 7.0, device="cuda") if lse else None
    uq.uniquan_attn_extend(T, n, H, c.n_kv, d, dev(q.reshape(T, H * d)).bfloat16(), dev(np.asarray(row_start, np.int32)),
                           dev(np.asarray(lens, np.int32)), scale=scale, O=O, row_lse=l, ws=workspace(T, n, H, c.n_kv, d, m),
                           mask=None if mask is None else words_of(mask, words),
                           pos=None if pos is None else dev(np.asarray(pos, np.int32)), window=window, sinks=sinks, **m)
    torch.cuda.synchronize()
    return O, l


def two_terms(T, n, H, n_kv):
    return -(-T // n) * (H // n_kv) <= 16


def check(c, m, q, row_start, lens, scale, what="", lse=True, **kw):
    """The call's results against the oracle's.  As kv_cases.attend_bounds, but where weights enter the second product
    as one bf16 value: 2^-8 of a weight times its value's size, of codes times the scale and their distance from the
    middle, at most 128 of 255 steps between a group's ends and so 1.004 of the largest value's size."""
    O, l = call(c, m, q, row_start, lens, scale, lse=lse, **kw)
    kw.pop("words", None)
    want, want_l, absv, absx, count = c.attend_rows(q, row_start, lens, scale, **kw)
    T, H, d = q.shape
    dx = (d + 8) * 2.0 ** -24 * WIDE[c.fmt] * absx
    term = 2.0 ** -14 if two_terms(T, len(lens), H, c.n_kv) else 1.01 * 2.0 ** -8
    rel = np.expm1(2 * dx) + term + (np.maximum(8, count)[:, None] + 8) * 2.0 ** -24 * WIDE[c.fmt]
    got = O.float().cpu().numpy().astype(np.float64).reshape(T, H, d)
    pad = np.isnan(want_l[:, 0])
    assert np.all(got[pad] == 7.0), f"{what}: padding written"
    empty = ~pad & (count == 0)
    assert np.all(got[empty] == 0), f"{what}: O of a row that sees nothing"
    bad = ~(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (rel * absv)[..., None] * 1.01)[~pad]
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off in O, NaN {np.isnan(got).sum()}, rows " \
        f"{np.unique(np.nonzero(~pad)[0][np.nonzero(bad)[0]])[:8]}"
    if lse:
        gl = l.cpu().numpy().astype(np.float64)
        assert np.all(gl[pad] == 7.0) and np.all(gl[empty] == -np.inf), f"{what}: lse of padding or of empty rows"
        live = ~pad & ~empty
        off = np.abs(gl[live] - want_l[live])
        tol = 1.4427 * dx[live] + 2.0 ** -17 + 2.0 ** -22 * np.abs(want_l[live])
        assert np.all(off <= tol), f"{what}: lse off by {off.max()}"
    return O, l


def tree(rs, m, back=5):
    """Depths and masks (own bit set) of m drafts with drawn parents."""
    depth, path = [], []
    for i in range(m):
        up = int(rs.integers(max(-1, i - back), i))
        depth.append(0 if up < 0 else depth[up] + 1)
        path.append((0 if up < 0 else path[up]) | 1 << i)
    return depth, path
