"""CPU oracle for the paged key/value cache and the attention of one new token
over it (serving a block deployed with UniQuan_F, arXiv 2506.03781).

TEST INFRASTRUCTURE, under the same rules as ``oracle.uniquan``: it imports
nothing from the HIP library.

Decisions (codes, scales, offsets, rotated values) are a float32 mirror of the
C header's formulas, in the stated operation order, so they are compared bit
for bit; values and attention are float64.

* cache arrays: k, v [n_pages, H_kv, P, row] (uint16 bf16 bits, or uint8 codes),
  statistics uint16 [n_pages, H_kv, d / group, P, 2] (bf16 bits of scale, lo);
* page table int [n_seq, max_pages]; ids outside [0, n_pages) are no page.
"""
from __future__ import annotations

import numpy as np

F32, F64 = np.float32, np.float64
TOP = {"u8": 255, "u4": 15}
TINY = F32(2.0 ** -126)


def bits(x):
    return np.asarray(x, F32).view(np.uint32)


def bf16(x):
    """bf16 bits of fp32 x, to nearest even (NaN kept)."""
    b = bits(x).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint32)
    return np.where(np.isnan(x), 0x7FC0, r & 0xFFFF).astype(np.uint16)


def from_bf16(h):
    return (np.asarray(h, np.uint16).astype(np.uint32) << 16).view(F32)


def down(x):
    """fp32 x rounded towards -infinity to bf16 (as fp32)."""
    cut = (bits(x) >> 16 << 16).view(F32)
    return np.where(cut > x, ((bits(cut).astype(np.uint64) + 0x10000).astype(np.uint32)).view(F32), cut).astype(F32)


def up(x):
    """fp32 x >= 0 rounded towards +infinity to bf16 (as fp32)."""
    cut = (bits(x) >> 16 << 16).view(F32)
    return np.where(cut < x, ((bits(cut).astype(np.uint64) + 0x10000).astype(np.uint32)).view(F32), cut).astype(F32)


def encode(x, fmt, group):
    """Codes [..., d] and (scale, lo) fp32 [..., d / group] of fp32 x [..., d]."""
    x = np.asarray(x, F32)
    g = x.reshape(*x.shape[:-1], -1, group)
    top = F32(TOP[fmt])
    with np.errstate(all="ignore"):
        lo = down(g.min(-1))
        spread = (g.max(-1) - lo).astype(F32)
        bad = ~np.isfinite(g).all(-1) | ~np.isfinite(spread)
        sc = up(np.maximum(spread, F32(0)) * (F32(1) / top))
        sc = np.where(sc < TINY, F32(0), sc).astype(F32)
        inv = np.where(sc > 0, F32(1) / sc, F32(0)).astype(F32)
        c = np.rint((g - lo[..., None]) * inv[..., None])
        c = np.where(bad[..., None] | np.isnan(c), 0, np.clip(c, 0, TOP[fmt])).astype(np.uint8)
    nan = F32(np.nan)
    return c.reshape(x.shape), np.where(bad, nan, sc).astype(F32), np.where(bad, nan, lo).astype(F32)


def place(d, fmt, key):
    """Position of every channel's code in a row."""
    ch = np.arange(d)
    if not key:
        return ch % 16 * (d // 16) + ch // 16
    j = ch % 8 if fmt == "u8" else ch % 8 // 2 + 4 * (ch % 2)
    return ch // 8 % 4 * (d // 4) + 8 * (ch // 32) + j


def pack(codes, fmt, key):
    d = codes.shape[-1]
    row = np.zeros_like(codes)
    row[..., place(d, fmt, key)] = codes
    return row if fmt == "u8" else row[..., 0::2] | row[..., 1::2] << 4


def unpack(row, fmt, key):
    if fmt == "u4":
        row = np.stack([row & 15, row >> 4], -1).reshape(*row.shape[:-1], 2 * row.shape[-1])
    return row[..., place(row.shape[-1], fmt, key)]


def rotate(x, cs):
    """x [T, heads, d] fp32 rotated by cs [T, d / 2, 2]."""
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h], x[..., h:], cs[:, None, :, 0], cs[:, None, :, 1]
    return np.concatenate([a * c - b * s, b * c + a * s], -1).astype(F32)


class Cache:
    """The cache's arrays on the host."""

    def __init__(self, n_pages, n_kv, d, P, fmt, group, table):
        self.n_pages, self.n_kv, self.d, self.P, self.fmt, self.group = n_pages, n_kv, d, P, fmt, group
        self.table = np.asarray(table, np.int64)
        shape = (n_pages, n_kv, P, d // 2 if fmt == "u4" else d)
        dt = np.uint16 if fmt == "bf16" else np.uint8
        self.k, self.v = np.zeros(shape, dt), np.zeros(shape, dt)
        self.k_stat = self.v_stat = None
        if fmt != "bf16":
            self.k_stat, self.v_stat = (np.zeros((n_pages, n_kv, d // group, P, 2), np.uint16) for _ in range(2))

    def page(self, s, pos):
        """Page of a position, or -1."""
        if not (0 <= s < self.table.shape[0] and 0 <= pos < self.table.shape[1] * self.P):
            return -1
        p = self.table[s, pos // self.P]
        return int(p) if 0 <= p < self.n_pages else -1

    def put(self, key, page, r, x):
        """fp32 rows x [n_kv, d] to place r of a page."""
        buf, stat = (self.k, self.k_stat) if key else (self.v, self.v_stat)
        if self.fmt == "bf16":
            buf[page, :, r] = bf16(x)
            return
        c, sc, lo = encode(x, self.fmt, self.group)
        buf[page, :, r] = pack(c, self.fmt, key)
        stat[page, :, :, r, 0] = np.where(np.isnan(sc), 0x7FC0, bits(sc) >> 16)
        stat[page, :, :, r, 1] = np.where(np.isnan(lo), 0x7FC0, bits(lo) >> 16)

    def append(self, k, v, pos, q=None, q_out=None, seq=None, cs=None):
        """Rows k, v [T, n_kv, d] fp32 (q [T, H, d] to q_out bf16 bits), as the C header states."""
        for t in range(len(pos)):
            s, p = t if seq is None else int(seq[t]), int(pos[t])
            if p < 0 or p >= self.table.shape[1] * self.P or not 0 <= s < self.table.shape[0]:
                continue
            if cs is not None and p >= len(cs):
                continue
            turn = (lambda x: rotate(x[None], cs[p:p + 1])[0]) if cs is not None else (lambda x: x)
            if q is not None:
                q_out[t] = bf16(turn(q[t])).reshape(q_out[t].shape)
            page = self.page(s, p)
            if page >= 0:
                self.put(True, page, p % self.P, turn(k[t]))
                self.put(False, page, p % self.P, v[t])

    def values(self, key, page, r):
        """fp32 values [n_kv, d] of place r of a page: lo + scale c, in that order."""
        buf, stat = (self.k, self.k_stat) if key else (self.v, self.v_stat)
        if self.fmt == "bf16":
            return from_bf16(buf[page, :, r])
        c = unpack(buf[page, :, r], self.fmt, key).astype(F32).reshape(self.n_kv, -1, self.group)
        st = from_bf16(stat[page, :, :, r])
        with np.errstate(all="ignore"):
            return (st[..., 1:] + st[..., :1] * c).astype(F32).reshape(self.n_kv, self.d)

    def read(self, lens, L, start=None):
        """K, V fp32 [n_kv, n_seq, L, d]."""
        n = self.table.shape[0]
        K, V = (np.zeros((self.n_kv, n, L, self.d), F32) for _ in range(2))
        for s in range(n):
            for i in range(L):
                p = i + (0 if start is None else int(start[s]))
                page = self.page(s, p) if 0 <= p < lens[s] else -1
                if page >= 0:
                    K[:, s, i], V[:, s, i] = (self.values(key, page, p % self.P) for key in (True, False))
        return K, V

    def held(self, s, n):
        """Pages and places of sequence s's first n positions that lie on a page."""
        at = [(self.page(s, p), p % self.P) for p in range(min(int(n), self.table.shape[1] * self.P))]
        at = np.array([a for a in at if a[0] >= 0], np.int64).reshape(-1, 2)
        return at[:, 0], at[:, 1]

    def dense(self, s, n):
        """K, V float64 [n_kv, positions, d] of those."""
        page, r = self.held(s, n)
        out = []
        for key in (True, False):
            buf, stat = (self.k, self.k_stat) if key else (self.v, self.v_stat)
            rows = buf[page, :, r]                                  # [positions, n_kv, row]
            if self.fmt == "bf16":
                x = from_bf16(rows).astype(F64)
            else:
                c = unpack(rows, self.fmt, key).astype(F64).reshape(len(page), self.n_kv, self.d // self.group, self.group)
                st = from_bf16(stat[page, :, :, r]).astype(F64)
                x = (st[..., 1:] + st[..., :1] * c).reshape(len(page), self.n_kv, self.d)
            out.append(x.transpose(1, 0, 2))
        return out

    def attend(self, q, lens, scale):
        """O float64 [n, H, d], base-2 log-sum-exp [n, H] of bf16-valued q [n, H, d]; and for error bounds
        sum_t p_t max_i |v_ti| and max_t scale max_i |k_ti| sum_i |q_i| [n, H]."""
        n, H, d = q.shape
        O, lse = np.zeros((n, H, d)), np.full((n, H), -np.inf)
        absv, absx = np.zeros((n, H)), np.zeros((n, H))
        for s in range(n):
            K, V = self.dense(s, lens[s])
            if K.shape[1] == 0:
                continue
            for h in range(H):
                g = h // (H // self.n_kv)
                x = scale * (K[g] @ q[s, h].astype(F64))
                m = x.max()
                p = np.exp(x - m)
                lse[s, h] = (m + np.log(p.sum())) / np.log(2.0)
                p /= p.sum()
                O[s, h] = p @ V[g]
                absv[s, h] = p @ np.abs(V[g]).max(-1)
                absx[s, h] = abs(scale) * np.abs(K[g]).max() * np.abs(q[s, h]).sum()
        return O, lse, absv, absx

    def attend_rows(self, q, row_start, lens, scale, mask=None, pos=None, window=0, sinks=0):
        """attend for several rows per sequence (uniquan_attn_extend): q [T, H, d] bf16 values, mask a list of T
        Python integers.  Rows of no sequence are NaN.  Also the number of positions that each row sees."""
        T, H, d = q.shape
        O, lse = np.full((T, H, d), np.nan), np.full((T, H), np.nan)
        absv, absx, count = np.zeros((T, H)), np.zeros((T, H)), np.zeros(T, int)
        cap = self.table.shape[1] * self.P
        for s in range(self.table.shape[0]):
            first, m = int(row_start[s]), int(row_start[s + 1]) - int(row_start[s])
            if m == 0:
                continue
            at = np.array([p for p in range(max(0, min(int(lens[s]), cap))) if self.page(s, p) >= 0], np.int64)
            K, V = self.dense(s, max(0, int(lens[s])))
            base = max(int(lens[s]), 0) - m
            for j in range(m):
                r = first + j
                P = base + j if pos is None else int(pos[r])
                near = (at > P - window) | (at < sinks) if window else np.ones(len(at), bool)
                if mask is None:
                    see = near & (at <= base + j)
                else:
                    see = np.array([bool(near[i]) if t < base else bool(mask[r] >> int(t - base) & 1)
                                    for i, t in enumerate(at)], bool).reshape(-1)
                count[r] = see.sum()
                O[r], lse[r] = 0, -np.inf
                if not see.any():
                    continue
                for h in range(H):
                    g = h // (H // self.n_kv)
                    k, v = K[g][see], V[g][see]
                    x = scale * (k @ q[r, h].astype(F64))
                    top = x.max()
                    p = np.exp(x - top)
                    lse[r, h] = (top + np.log(p.sum())) / np.log(2.0)
                    p /= p.sum()
                    O[r, h] = p @ v
                    absv[r, h] = p @ np.abs(v).max(-1)
                    absx[r, h] = abs(scale) * np.abs(k).max() * np.abs(q[r, h]).sum()
        return O, lse, absv, absx, count
