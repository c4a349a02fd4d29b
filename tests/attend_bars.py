"""Bars for uniquan_attn_decode that a lost, doubled or misplaced block of
positions breaks (test_attend_bars.py shows that on the host), and caches whose
answer shows each block.  kv_cases.attend_bounds multiplies the largest key
channel by sum |q|, which for codes and rows of thousands of positions is more
than the answer itself.

Per position t, with u = 2^-24 and magnitudes counted as the kernel adds them:

  A_t = |scale| sum_i |q_i| K_ti,  K the key's magnitude: |k| of bf16, scale c + |lo| of codes
  V_ti  the value's magnitude: |v| of bf16, scale |c - middle| + |scale middle + lo| of codes (middle 128 or 8)

Errors, relative to a weight:
  its score     d + 8 roundings of sums up to A_t, taken as independent and four standard deviations of their sum
                (a rounding's is u / sqrt(3)): 4 sqrt((d + 8) / 3) u A_t, twice, as the weights' sum has it too
  its two terms in the product with the values: 2^-15
  exp2 (1 ulp, and its argument rounded below 32: 2^-20) and the running rescales: 2^-18
  the sums over n positions: 4 sqrt((n + 64) / 3) u, as above
so |O - exact| <= sum_t p_t rel_t (V_ti + |O_i|), and half a bf16 step of O.  The same normwise per row and head.
"""
import numpy as np
import torch

import oracle.kv_cache as KV
from kv_cases import F32, dev, group_of, on_device, poison, rounded, tables
from paper_2506_03781_amd import uniquan as uq

BLOCK = 128  # positions of a workgroup's round
MID = {"u8": 128, "u4": 8}


def magnitudes(c, s, n, key):
    """[n_kv, positions, d] of sequence s's first n positions, as above."""
    page, r = c.held(s, n)
    buf, stat = (c.k, c.k_stat) if key else (c.v, c.v_stat)
    if c.fmt == "bf16":
        return np.abs(KV.from_bf16(buf[page, :, r]).astype(np.float64)).transpose(1, 0, 2)
    codes = KV.unpack(buf[page, :, r], c.fmt, key).astype(np.float64).reshape(len(page), c.n_kv, -1, c.group)
    st = KV.from_bf16(stat[page, :, :, r]).astype(np.float64)
    sc, lo = st[..., :1], st[..., 1:]
    x = sc * codes + np.abs(lo) if key else sc * np.abs(codes - MID[c.fmt]) + np.abs(sc * MID[c.fmt] + lo)
    return x.reshape(len(page), c.n_kv, c.d).transpose(1, 0, 2)


def bars(c, q, lens, scale):
    """O [n, H, d] in 64 bits, its bar element by element, and its bar normwise [n, H]."""
    n, H, d = q.shape
    O, tol, norm = np.zeros((n, H, d)), np.zeros((n, H, d)), np.zeros((n, H))
    u = 2.0 ** -24
    for s in range(n):
        K, V = c.dense(s, lens[s])
        if K.shape[1] == 0:
            continue
        Ka, Va = (magnitudes(c, s, lens[s], key) for key in (True, False))
        for h in range(H):
            g = h // (H // c.n_kv)
            qh = q[s, h].astype(np.float64)
            x = scale * (K[g] @ qh)
            p = np.exp(x - x.max())
            p /= p.sum()
            dx = 4 * np.sqrt((d + 8) / 3) * u * abs(scale) * (Ka[g] @ np.abs(qh))
            rel = np.expm1(2 * dx) + 2.0 ** -15 + 2.0 ** -18 + 4 * np.sqrt((len(p) + 64) / 3) * u
            O[s, h] = p @ V[g]
            part = (p * rel) @ (Va[g] + np.abs(O[s, h]))
            tol[s, h] = 2.0 ** -8 * np.abs(O[s, h]) + part
            norm[s, h] = 2.0 ** -8 * np.linalg.norm(O[s, h]) + np.linalg.norm(part)
    return O, tol, norm


def broken(got, c, q, lens, scale, want=None):
    """Whether got [n, H, d] breaks a bar: element by element, normwise (each [n, H])."""
    O, tol, norm = bars(c, q, lens, scale) if want is None else want
    return (~(np.abs(got - O) <= tol)).any(-1), ~(np.linalg.norm(got - O, axis=-1) <= norm)


def store(c, key, s, p, x):
    """Rows x [positions, n_kv, d] at sequence s's positions p, as Cache.put does one by one."""
    page, r = c.table[s, p // c.P], p % c.P
    buf, stat = (c.k, c.k_stat) if key else (c.v, c.v_stat)
    if c.fmt == "bf16":
        buf[page, :, r] = KV.bf16(x)
        return
    codes, sc, lo = KV.encode(x, c.fmt, c.group)
    buf[page, :, r] = KV.pack(codes, c.fmt, key)
    stat[page, :, :, r, 0], stat[page, :, :, r, 1] = KV.bits(sc) >> 16, KV.bits(lo) >> 16


def block_values(p, n_kv, d):
    """Values of positions p that show their blocks: 1 in one channel a head, no two blocks of a row in the same."""
    v = np.zeros((len(p), n_kv, d), F32)
    h = np.arange(n_kv)
    v[np.arange(len(p))[:, None], h, (p[:, None] // BLOCK + 7 * h) % d] = 1
    return v


def long_rows(rs, lens, n_kv, d, P, fmt, group, shown):
    """A cache of long rows: keys of order one whose scores differ by block (along a channel in which the queries are
    8 sqrt(d) / d), values that show their block or drawn ones."""
    t, n_pages = tables(rs, lens, P)
    c = KV.Cache(n_pages, n_kv, d, P, fmt, group_of(group, d) if fmt != "bf16" else 0, t)
    poison(c)
    for s, ln in enumerate(lens):
        if ln == 0:
            continue
        p = np.arange(int(ln))
        k, v = (rs.standard_normal((ln, n_kv, d)).astype(F32) for _ in range(2))
        k[:, :, 3] = (p // BLOCK % 3 - 1)[:, None]
        store(c, True, s, p, k)
        store(c, False, s, p, block_values(p, n_kv, d) if shown else v)
    return c


def queries(rs, n, H, d):
    q = rounded(rs, n, H, d)
    q[..., 3] = KV.from_bf16(KV.bf16(np.float32(d ** 0.5)))
    return q


LONG = [5000, 3, 0, 2049, 777, 4097]


def attend(c, q, lens, scale):
    """O [n, H, d] and the log-sum-exp [n, H] from the device, in 64 bits."""
    n, H, d = q.shape
    m = on_device(c)
    O = torch.full((n, H * d), float("nan"), device="cuda", dtype=torch.bfloat16)
    lse = torch.full((n, H), float("nan"), device="cuda")
    ws = torch.full((max(1, uq.uniquan_attn_decode_ws(n, H, c.n_kv, d, m["table"].shape[1], c.P)),), float("nan"),
                    device="cuda")
    uq.uniquan_attn_decode(n, H, c.n_kv, d, dev(q.reshape(n, H * d)).bfloat16(), dev(np.asarray(lens, np.int32)),
                           scale=scale, O=O, row_lse=lse, ws=ws, **m)
    torch.cuda.synchronize()
    return O.float().cpu().numpy().astype(np.float64).reshape(n, H, d), lse.cpu().numpy().astype(np.float64)
