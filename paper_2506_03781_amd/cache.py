"""The paged key/value cache of one attention module: what a serving loop
keeps between the decoding steps of a deployed block.

One step of a block on T rows, one per sequence, is

    add_rmsnorm, the query, key and value products (uniquan_bcq_matmul, fp32 rows)
    cache.append(k, v, pos, q=q, q_out=Qr, cs=table)    rotated, stored
    cache.attend(Qr, lens, O)                           O: the output product's bf16 rows
    uniquan_bcq_matmul(O), then the MLP module

and a prompt is appended in the same way, its rows naming their sequences;
``read`` gives it back in the layout of ``uniquan_attn_fwd``.  That attention
takes d = 128, as many queries as keys and multiples of 32 positions: a whole
prompt (padded behind its end), not a part of one behind positions that are
cached already, nor heads of 64 channels; those are attended one token at a time.

The rotary table cs [n, d / 2, 2] holds (cos, sin) of every position.
``uniquan_rope_table`` makes its angles in fp32, off by up to p 2^-23 at position
p; a table for tens of thousands of positions is made in 64 bits:

    a = torch.arange(n, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    cs = torch.stack([a.cos(), a.sin()], -1).float().cuda()

All arithmetic runs in libuniquan.so; torch only allocates device memory.
"""
from __future__ import annotations

import torch

from . import uniquan as uq

FORMATS = {"bf16": uq.KV_BF16, "u8": uq.KV_U8, "u4": uq.KV_U4}


class KVCache:
    """n_pages pages of page_len positions of n_kv key/value heads of d
    channels, stored as "bf16", "u8" or "u4" (codes with a scale and an offset
    for every `group` channels: 32 or d, the default).  `table` [n_seq,
    max_pages] (int32) names the pages of each sequence, -1 where there is
    none; the caller fills it and keeps each sequence's length."""

    def __init__(self, n_pages, n_kv, n_seq, max_pages, d=128, page_len=64, fmt="bf16", group=None, device="cuda"):
        self.n_pages, self.n_kv, self.d, self.page_len = n_pages, n_kv, d, page_len
        self.fmt = FORMATS[fmt]
        self.group = 0 if fmt == "bf16" else d if group is None else group
        row = d // 2 if fmt == "u4" else d
        dt = torch.bfloat16 if fmt == "bf16" else torch.uint8
        z = torch.zeros
        self.k, self.v = (z(n_pages, n_kv, page_len, row, dtype=dt, device=device) for _ in range(2))
        self.k_stat = self.v_stat = None
        if self.group:
            self.k_stat, self.v_stat = (z(n_pages, n_kv, d // self.group, page_len, 2, dtype=torch.bfloat16,
                                          device=device) for _ in range(2))
        self.table = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=device)

    def _form(self):
        return dict(fmt=self.fmt, group=self.group, page_len=self.page_len, k_stat=self.k_stat, v_stat=self.v_stat)

    def append(self, k, v, pos, q=None, q_out=None, seq=None, cs=None, stream=None):
        """Rows k, v [T, n_kv d] at positions pos [T] of sequences seq [T] (None: row t of sequence t); q [T, H d]
        to q_out; q and k rotated by cs where given."""
        H = self.n_kv if q is None else q.shape[1] // self.d
        uq.uniquan_kv_append(k.shape[0], H, self.n_kv, self.d, q, k, v, pos, self.table, self.k, self.v, q_out, seq=seq,
                             cs=cs, stream=stream, **self._form())

    def read(self, lens, L, K, V, start=None, stream=None):
        """Positions start[s] .. + L of every sequence into K, V [n_kv, n_seq, L, d] (fp32 or bf16)."""
        uq.uniquan_kv_read(self.table.shape[0], self.n_kv, self.d, L, lens, self.table, self.k, self.v, K, V,
                           start=start, stream=stream, **self._form())

    def workspace(self, H):
        """An fp32 workspace for attend with H query heads (None: none needed).  Calls that may overlap, and
        graphs that are replayed at the same time, need one each."""
        need = uq.uniquan_attn_decode_ws(self.table.shape[0], H, self.n_kv, self.d, self.table.shape[1], self.page_len)
        return torch.empty(need, dtype=torch.float32, device=self.k.device) if need else None

    def attend(self, Q, lens, O, row_lse=None, scale=None, ws=None, stream=None):
        """O [n_seq, H d] = attention of the rows Q [n_seq, H d] over each sequence's first lens[s] positions.
        Without ws (from workspace()) the call takes one from torch on the current stream; a call on another
        stream or within uniquan.record, whose launches outlive it, brings its own."""
        n, H = self.table.shape[0], Q.shape[1] // self.d
        if ws is None:
            ws = self.workspace(H)
            if ws is not None and (stream is not None or uq._recorder is not None):
                raise ValueError("attend needs the caller's ws on a given stream and within record()")
        uq.uniquan_attn_decode(n, H, self.n_kv, self.d, Q, lens, self.table, self.k, self.v,
                               1.0 / float(self.d) ** 0.5 if scale is None else scale, O, row_lse, ws, stream=stream,
                               **self._form())
