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
prompt (padded behind its end).  For heads of 64 channels, and for a part of a
prompt behind positions that are cached already, ``extend`` attends to the cache.

A step that verifies a tree of drafted tokens, m rows of a sequence whose length
counts them (the drafts' places are the last m, their positions base + depth):

    cache.append(k, v, place, q=q, q_out=Qr, seq=seq, cs=table, rot=position, axis=zeros)
    cache.extend(Qr, row_start, lens, O, mask=ancestors)
    ...                                                 the rest of the model
    uniquan_sample(logits, u, token)                    a token after every draft

and the drafts of the path that agrees are appended again, from the products'
rows that the caller has kept, at places that are their positions.

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

    def append(self, k, v, pos, q=None, q_out=None, seq=None, cs=None, stream=None, rot=None, axis=None):
        """Rows k, v [T, n_kv d] at positions pos [T] of sequences seq [T] (None: row t of sequence t); q [T, H d]
        to q_out; q and k rotated by cs where given: at pos, or, with rot [T, n_axes] and axis [d / 2], pair i at
        rot[t, axis[i]] (drafted tokens whose place is not their position, images and videos)."""
        H = self.n_kv if q is None else q.shape[1] // self.d
        rows = (k.shape[0], H, self.n_kv, self.d, q, k, v, pos)
        if (rot is None) != (axis is None):
            raise ValueError("rot and axis must be given together")
        if rot is None:
            uq.uniquan_kv_append(*rows, self.table, self.k, self.v, q_out, seq=seq, cs=cs, stream=stream, **self._form())
        else:
            uq.uniquan_kv_append_axes(*rows, rot, axis, cs, self.table, self.k, self.v, q_out, seq=seq, stream=stream,
                                      **self._form())

    def read(self, lens, L, K, V, start=None, stream=None):
        """Positions start[s] .. + L of every sequence into K, V [n_kv, n_seq, L, d] (fp32 or bf16)."""
        uq.uniquan_kv_read(self.table.shape[0], self.n_kv, self.d, L, lens, self.table, self.k, self.v, K, V,
                           start=start, stream=stream, **self._form())

    def workspace(self, H, rows=None):
        """An fp32 workspace for attend with H query heads, or for extend with `rows` rows (None: none needed).
        Calls that may overlap, and graphs that are replayed at the same time, need one each."""
        n, size = self.table.shape[0], (H, self.n_kv, self.d, self.table.shape[1], self.page_len)
        need = uq.uniquan_attn_decode_ws(n, *size) if rows is None else uq.uniquan_attn_extend_ws(rows, n, *size)
        return torch.empty(need, dtype=torch.float32, device=self.k.device) if need else None

    def _own_ws(self, ws, stream, name):
        if ws is not None and (stream is not None or uq._recorder is not None):
            raise ValueError(f"{name} needs the caller's ws on a given stream and within record()")
        return ws

    def attend(self, Q, lens, O, row_lse=None, scale=None, ws=None, stream=None):
        """O [n_seq, H d] = attention of the rows Q [n_seq, H d] over each sequence's first lens[s] positions.
        Without ws (from workspace()) the call takes one from torch on the current stream; a call on another
        stream or within uniquan.record, whose launches outlive it, brings its own."""
        n, H = self.table.shape[0], Q.shape[1] // self.d
        if ws is None:
            ws = self._own_ws(self.workspace(H), stream, "attend")
        uq.uniquan_attn_decode(n, H, self.n_kv, self.d, Q, lens, self.table, self.k, self.v,
                               1.0 / float(self.d) ** 0.5 if scale is None else scale, O, row_lse, ws, stream=stream,
                               **self._form())

    def extend(self, Q, row_start, lens, O, row_lse=None, mask=None, pos=None, window=0, sinks=0, scale=None, ws=None,
               stream=None):
        """O [T, H d] = attention of the rows Q [T, H d], row_start[s] .. row_start[s + 1] of them of sequence s, at
        the last of its lens[s] places: parts of prompts, and with mask [T, words] trees of drafts; window and sinks
        as in uniquan_attn_extend.  ws (from workspace(H, rows=T)) as for attend."""
        n, T, H = self.table.shape[0], Q.shape[0], Q.shape[1] // self.d
        if ws is None:
            ws = self._own_ws(self.workspace(H, T), stream, "extend")
        uq.uniquan_attn_extend(T, n, H, self.n_kv, self.d, Q, row_start, lens, self.table, self.k, self.v,
                               1.0 / float(self.d) ** 0.5 if scale is None else scale, O, row_lse, ws, mask=mask, pos=pos,
                               window=window, sinks=sinks, stream=stream, **self._form())
