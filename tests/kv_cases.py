"""Shared by the tests of the paged key/value cache: seeded caches on the host
(oracle.kv_cache) and on the device, with everything that no sequence holds
filled with NaN."""
import numpy as np
import torch

import oracle.kv_cache as KV
from paper_2506_03781_amd import uniquan as uq

F32 = np.float32
FMT = {"bf16": uq.KV_BF16, "u8": uq.KV_U8, "u4": uq.KV_U4}
FORMS = [("bf16", 0), ("u8", 32), ("u8", None), ("u4", 32), ("u4", None)]  # None: one group a head


def group_of(group, d):
    return d if group is None else group


def rounded(rs, *shape):
    """Standard normal values that bf16 holds."""
    return KV.from_bf16(KV.bf16(rs.standard_normal(shape).astype(F32)))


def tables(rs, lens, P, spare=2, max_pages=None):
    """Page table [n, max_pages] with the pages in a drawn order, -1 behind each sequence's last; page count."""
    need = [-(-int(ln) // P) for ln in lens]
    mp = max(1, max(need, default=1)) if max_pages is None else max_pages
    n_pages = sum(need) + spare
    order = rs.permutation(n_pages)
    t = np.full((len(lens), mp), -1)
    at = 0
    for s, n in enumerate(need):
        t[s, :n] = order[at:at + n]
        at += n
    return t, n_pages


def poison(c):
    """Every byte of the cache set: NaN where values or statistics lie."""
    for a in (c.k, c.v):
        a[...] = 0x7FC1 if a.dtype == np.uint16 else 0xFF
    if c.k_stat is not None:
        c.k_stat[...] = 0x7FC1
        c.v_stat[...] = 0x7FC1


def filled(rs, lens, n_kv, d, P, fmt, group, max_pages=None, outlier=True, table=None):
    """Host cache holding lens[s] drawn positions of every sequence, NaN elsewhere."""
    t, n_pages = tables(rs, lens, P, max_pages=max_pages) if table is None else table
    c = KV.Cache(n_pages, n_kv, d, P, fmt, group_of(group, d) if fmt != "bf16" else 0, t)
    poison(c)
    f = np.ones(d, F32)
    if outlier:
        f[rs.integers(d)] = 10
    for s, ln in enumerate(lens):
        for p in range(int(ln)):
            page = c.page(s, p)
            if page >= 0:
                c.put(True, page, p % P, (rs.standard_normal((n_kv, d)) * f).astype(F32))
                c.put(False, page, p % P, rs.standard_normal((n_kv, d)).astype(F32))
    return c


def dev(a, dtype=None):
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16)
    t = torch.from_numpy(a).cuda()
    return t if dtype is None else t.to(dtype)


def on_device(c):
    """The cache's arrays, page table and form as the binding takes them."""
    return dict(table=dev(c.table.astype(np.int32)), k_cache=dev(c.k), v_cache=dev(c.v),
                k_stat=None if c.k_stat is None else dev(c.k_stat), v_stat=None if c.v_stat is None else dev(c.v_stat),
                fmt=FMT[c.fmt], group=c.group, page_len=c.P)


def host_bits(t):
    """A device tensor's bits (bf16 as uint16)."""
    t = t.detach().cpu()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.numpy()


def same_cache(m, c, what=""):
    """The device cache equals the host's bit for bit; a NaN statistic may be any NaN."""
    for name, ref in (("k_cache", c.k), ("v_cache", c.v)):
        assert np.array_equal(host_bits(m[name]), ref), f"{what}: {name}"
    for name, ref in (("k_stat", c.k_stat), ("v_stat", c.v_stat)):
        if ref is not None:
            got = host_bits(m[name])
            nan = np.isnan(KV.from_bf16(ref))
            assert np.array_equal(np.isnan(KV.from_bf16(got)), nan), f"{what}: {name} NaN"
            assert np.array_equal(got[~nan], ref[~nan]), f"{what}: {name}"


def cos_sin(n, d):
    i = np.arange(d // 2)
    a = np.arange(n)[:, None] * 1e4 ** (-2.0 * i / d)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(F32)


# A sum over codes adds up code values, counted from 0, and takes their part of the offset away again: at most this
# many times the largest value, counting both.
WIDE = {"bf16": 1.0, "u8": 4.0, "u4": 4.0}


def attend_bounds(c, q, lens, scale):
    """O and log-sum-exp in 64 bits, and how far the kernel's may be off, element by element.

    With u = 2^-24 and d + 8 terms a score is off by dx = (d + 8) u WIDE max|x|, x = scale sum |q||k| (fp32 sums of
    exact products; the scaling and the exponent's argument are among the 8), so every weight by a factor within
    e^(2 dx).  Its exp2, the running rescales and its two bf16 terms in the product with the values: 2^-14.  The fp32
    sum over n values: (n + 8) u WIDE of sum p max|v| in the worst case.  O is then rounded to bf16 (half a step: 2^-8
    of the value).  log-sum-exp: log2(e) dx, and 2^-17 + 2^-22 of the value for the sum, its logarithm and the addition."""
    O, lse, absv, absx = c.attend(q, lens, scale)
    dx = (q.shape[-1] + 8) * 2.0 ** -24 * WIDE[c.fmt] * absx
    n = max(8, max(int(x) for x in lens))
    rel = np.expm1(2 * dx) + 2.0 ** -14 + (n + 8) * 2.0 ** -24 * WIDE[c.fmt]
    tol_l = 1.4427 * dx + 2.0 ** -17 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))
    return O, lse, 2.0 ** -8 * np.abs(O) + (rel * absv)[..., None] * 1.01, tol_l


def check_attend(got_O, got_lse, c, q, lens, scale, what=""):
    O, lse, tol_o, tol_l = attend_bounds(c, q, lens, scale)
    o = got_O.float().cpu().numpy().astype(np.float64).reshape(O.shape)
    empty = ~np.isfinite(lse)
    assert np.all(o[empty] == 0), f"{what}: O of an empty row"
    bad = ~(np.abs(o - O) <= tol_o)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off in O, NaN {np.isnan(o).sum()}"
    if got_lse is not None:
        gl = got_lse.cpu().numpy().astype(np.float64).reshape(lse.shape)
        assert np.all(gl[empty] == -np.inf), f"{what}: lse of an empty row"
        bad = ~(np.abs(gl[~empty] - lse[~empty]) <= tol_l[~empty])
        assert not bad.any(), f"{what}: lse off by {np.abs(gl[~empty] - lse[~empty]).max()}"
