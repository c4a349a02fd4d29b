"""The serving operators around the deployed products: a paged key/value cache,
written and read back, and the attention of one new token over it.

Kinds of case:

* append  new tokens into the cache (``uniquan_kv_append``): the queries and
          keys rotated at their positions, keys and values stored as bf16 or
          as 8- or 4-bit codes with a scale and an offset per group.  A bf16
          cache is returned as it stands; of a cache of codes, the new tokens
          are read back (``uniquan_kv_read``), as a prompt does whose own
          attention is to see the stored values.
* read    positions [start, start + L) of every sequence back as dense
          head-major arrays (``uniquan_kv_read``).
* attn    one query row per sequence over its pages
          (``uniquan_attn_decode``).

A case is a batch of n sequences.  ``ragged`` lengths spread over 0..L, one
sequence in eight idle (length 0); ``holes`` takes every fourth page out of
the page tables (an evicted page holds nothing); ``pad`` marks the last
eighth of an append's rows as padding.  Pages lie in the cache in an order
drawn from the seed.  Keys have 1% of their channels ten times the others'.

Stored forms.  A group of values (32 channels, or the whole head) with
minimum m and maximum M has lo = m rounded down to bf16 and
scale = (M - lo) / top rounded up to bf16 (top = 255 or 15); a code stands for
lo + scale code.  Keys' codes lie in a row by (channel / 8) % 4, then channel / 32,
then channel % 8; values' by channel % 16, then channel / 16; a byte holds two
4-bit codes, the lower one first, keys' eight of one run in the order
0 2 4 6 1 3 5 7.
"""
from __future__ import annotations

import math

import torch

own = False

KV = {"bf16": 0, "u8": 1, "u4": 2}
TOP = {"u8": 255, "u4": 15}
RUN = [0, 2, 4, 6, 1, 3, 5, 7]  # channels of a run of eight in the order of a 4-bit key row


def listed():
    return [
        # The smallest call: one user's first tokens, a 7B block's 32 heads.  Launches and latency.
        dict(name="attn_one_short", kind="attn", n=1, L=100, H=32, Hkv=32, d=128, fmt="bf16", group=0, page=16,
             ragged=False, holes=False),
        # The bench's 7B block (4 sequences of 2048 tokens, as many key/value heads as heads) one token later.
        dict(name="attn_7b_mha", kind="attn", n=4, L=2048, H=32, Hkv=32, d=128, fmt="bf16", group=0, page=64,
             ragged=False, holes=False),
        # A serving batch of unequal lengths, eight key/value heads, 8-bit codes.
        dict(name="attn_ragged_u8", kind="attn", n=48, L=8192, H=32, Hkv=8, d=128, fmt="u8", group=128, page=32,
             ragged=True, holes=False),
        # One very long document, 64 heads on 8, 4-bit codes in groups of 32: all the work in one row.
        dict(name="attn_long_u4", kind="attn", n=1, L=100001, H=64, Hkv=8, d=128, fmt="u4", group=32, page=256,
             ragged=False, holes=False),
        # The largest: 64 users of a 70B block (64 heads on 8), up to 16384 tokens each.
        dict(name="attn_70b_large", kind="attn", n=64, L=16384, H=64, Hkv=8, d=128, fmt="bf16", group=0, page=64,
             ragged=True, holes=False),
        # A small model's heads of 64 in sevens, small pages, evicted pages.
        dict(name="attn_d64_holes", kind="attn", n=33, L=1500, H=28, Hkv=4, d=64, fmt="u4", group=64, page=16,
             ragged=True, holes=True),
        # One new token of one user.
        dict(name="append_one", kind="append", n=1, tokens=1, start=517, H=32, Hkv=32, d=128, fmt="bf16", group=0,
             page=64, dtype="f32", pad=False, stacked=False),
        # One new token of 256 users, from the stacked key/value product's fp32 rows.
        dict(name="append_step_u4", kind="append", n=256, tokens=1, start=1000, H=64, Hkv=8, d=128, fmt="u4", group=32,
             page=64, dtype="f32", pad=False, stacked=True),
        # The bench's four 2048-token samples as prompts, grouped-query heads.
        dict(name="append_prompt_u8", kind="append", n=4, tokens=2048, start=0, H=32, Hkv=8, d=128, fmt="u8",
             group=128, page=64, dtype="bf16", pad=False, stacked=False),
        # Parts of prompts that start and end inside pages, heads of 64, a padded batch.
        dict(name="append_part_d64", kind="append", n=3, tokens=701, start=37, H=16, Hkv=16, d=64, fmt="bf16", group=0,
             page=16, dtype="f32", pad=True, stacked=True),
        # A prompt's keys and values back for its attention.
        dict(name="read_prompt_u8", kind="read", n=4, L=2048, start=0, Hkv=8, d=128, fmt="u8", group=32, page=64,
             out="bf16", ragged=True),
        # A long cache back in fp32, from an odd position on.
        dict(name="read_long_u4", kind="read", n=2, L=50001, start=11, Hkv=8, d=128, fmt="u4", group=32, page=128,
             out="f32", ragged=False),
    ]


# ---------------------------------------------------------------------------
# draw: one more case of the same ranges
# ---------------------------------------------------------------------------
MOST_ATTN = 64 * 16384 * 8 * 128       # values of K (or V) of the largest listed attention, padded
MOST_ATTN_BYTES = 2 * MOST_ATTN        # their bytes at half of the padded length (ragged), K and V, bf16
MOST_ROWS = 2 * 50001 * 8 * 128        # values of K (or V) of the largest listed read


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cache(rng):
    d = rng.choice([128, 128, 128, 64])
    fmt = rng.choice(["bf16", "u8", "u4"])
    return dict(Hkv=rng.choice([1, 2, 4, 8, 8, 16, 32]), d=d, fmt=fmt,
                group=0 if fmt == "bf16" else rng.choice([32, d]), page=rng.choice([16, 32, 64, 128, 256]))


def draw(rng):
    while True:
        kind = rng.choice(["attn", "attn", "attn", "append", "append", "read"])
        c = dict(kind=kind, **_cache(rng))
        if kind == "attn":
            c.update(n=_log(rng, 1, 256), L=_log(rng, 1, 100001), H=c["Hkv"] * rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16]),
                     ragged=rng.random() < 0.6, holes=rng.random() < 0.2)
            if c["H"] > 128 or c["n"] * c["L"] * c["Hkv"] * c["d"] > MOST_ATTN or work(c)["bytes"] > MOST_ATTN_BYTES:
                continue
        elif kind == "append":
            step = rng.random() < 0.4
            c.update(n=_log(rng, 1, 256) if step else _log(rng, 1, 8), tokens=1 if step else _log(rng, 2, 8192),
                     start=rng.choice([0, rng.randint(1, 2000)]), H=c["Hkv"] * rng.choice([1, 2, 4, 7, 8]),
                     dtype=rng.choice(["f32", "bf16"]), pad=rng.random() < 0.3, stacked=rng.random() < 0.5)
            if c["H"] > 128 or c["n"] * c["tokens"] * (c["H"] + 2 * c["Hkv"]) * c["d"] > 8192 * 96 * 128:
                continue
        else:
            c.update(n=_log(rng, 1, 64), L=_log(rng, 1, 50001), start=rng.choice([0, rng.randint(1, 500)]),
                     out=rng.choice(["f32", "bf16"]), ragged=rng.random() < 0.5)
            if c["n"] * c["L"] * c["Hkv"] * c["d"] > MOST_ROWS:
                continue
        return c


def _lens(c):
    """Lengths of an attn or read case's sequences."""
    end = c["L"] + c.get("start", 0)
    if not c["ragged"]:
        return [end] * c["n"]
    part = ((i * 0.6180339887498949) % 1.0 for i in range(c["n"]))
    return [0 if i % 8 == 5 else end - int(end * u) for i, u in enumerate(part)]


def _positions(c):
    """Sequence and position of an append case's rows; padding has position -1."""
    T, n, m = c["n"] * c["tokens"], c["n"], c["tokens"]
    row = torch.arange(T, device="cuda", dtype=torch.int32)
    pos = c["start"] + row % m
    if c["pad"]:
        pos = torch.where(row >= T - T // 8, -1, pos)
    return row // m, pos


def _hole(c, j):
    return bool(c.get("holes")) and j % 4 == 2


# ---------------------------------------------------------------------------
# the stored forms, in plain torch
# ---------------------------------------------------------------------------
def _down(x):
    """x rounded down to a bf16 value (as fp32)."""
    b = x.view(torch.int32) & -65536
    y = b.view(torch.float32)
    return torch.where(y > x, (b + 65536).view(torch.float32), y)


def _up(x):
    """x >= 0 rounded up to a bf16 value (as fp32)."""
    b = x.view(torch.int32) & -65536
    y = b.view(torch.float32)
    return torch.where(y < x, (b + 65536).view(torch.float32), y)


def _encode(x, fmt, group):
    """Codes [..., d] (int32) and (scale, lo) [..., d / group, 2] of x [..., d] fp32."""
    top = TOP[fmt]
    g = x.unflatten(-1, (-1, group))
    lo = _down(g.amin(-1))
    spread = g.amax(-1) - lo
    sc = _up((spread * (1.0 / top)).clamp(min=0))
    sc = torch.where(sc < 2.0 ** -126, torch.zeros_like(sc), sc)
    inv = torch.where(sc > 0, torch.ones_like(sc) / sc, torch.zeros_like(sc))
    code = torch.round((g - lo[..., None]) * inv[..., None]).clamp(0, top)
    bad = ~torch.isfinite(spread)
    nan = torch.full_like(sc, float("nan"))
    code = torch.where(bad[..., None], torch.zeros_like(code), code).int().flatten(-2)
    return code, torch.stack([torch.where(bad, nan, sc), torch.where(bad, nan, lo)], -1)


def _to_row(code, fmt, key):
    """A row's bytes [..., d or d / 2] from its codes [..., d]."""
    d = code.shape[-1]
    if key:
        code = code.unflatten(-1, (d // 32, 4, 8)).transpose(-3, -2)
        code = code[..., RUN] if fmt == "u4" else code
    else:
        code = code.unflatten(-1, (d // 16, 16)).transpose(-2, -1)
    code = code.reshape(*code.shape[:-3], d) if key else code.reshape(*code.shape[:-2], d)
    if fmt == "u4":
        code = code[..., 0::2] | code[..., 1::2] << 4
    return code.to(torch.uint8)


def _from_row(row, fmt, key):
    """Codes [..., d] from a row's bytes."""
    if fmt == "u4":
        row = torch.stack([row & 15, row >> 4], -1).flatten(-2)
    d = row.shape[-1]
    if not key:
        return row.unflatten(-1, (16, d // 16)).transpose(-2, -1).flatten(-2)
    row = row.unflatten(-1, (4, d // 32, 8))
    if fmt == "u4":
        row = row[..., [RUN.index(j) for j in range(8)]]
    return row.transpose(-3, -2).flatten(-3)


def _values(rows, stat, fmt, key):
    """fp32 values [..., P, d] of cache rows [..., P, row] with (scale, lo) in stat [..., d / group, P, 2]."""
    if fmt == "bf16":
        return rows.float()
    code = _from_row(rows, fmt, key).float()
    st = stat.float().transpose(-3, -2)                 # [..., P, d / group, 2]
    g = code.unflatten(-1, (st.shape[-2], -1))
    return (st[..., 1:] + st[..., :1] * g).flatten(-2)


def _store(x, fmt, group, key):
    """Cache rows and stat (None for bf16) of fp32 pages x [..., P, d]."""
    if fmt == "bf16":
        return x.bfloat16(), None
    code, st = _encode(x, fmt, group)
    return _to_row(code, fmt, key), st.transpose(-3, -2).bfloat16().contiguous()


def _row_bytes(c):
    """Bytes of one position of one head in K (or V), and of its scales and offsets."""
    d = c["d"]
    return (2 * d, 0) if c["fmt"] == "bf16" else (d if c["fmt"] == "u8" else d // 2, 4 * d // c["group"])


# ---------------------------------------------------------------------------
# prepare
# ---------------------------------------------------------------------------
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 1009 + salt)


def _normal(seed, salt, *shape):
    return torch.randn(*shape, generator=_gen(seed, salt), device="cuda")


def _outliers(seed, salt, width):
    """Channel factors: ten for 1% of them (one at least), else one."""
    f = torch.ones(width, device="cuda")
    f[torch.randperm(width, generator=_gen(seed, salt), device="cuda")[:max(1, width // 100)]] = 10.0
    return f


def _tables(c, seed, lens):
    """Page table and the number of pages of the cache, three of them no sequence's."""
    P, n = c["page"], c["n"]
    per = max(1, max((ln + P - 1) // P for ln in lens))
    n_pages = n * per + 3
    order = torch.randperm(n_pages, generator=_gen(seed, 1), device="cuda")[:n * per].int()
    table = order.reshape(n, per)
    if c.get("holes"):
        table = torch.where(torch.tensor([_hole(c, j) for j in range(per)], device="cuda"), -1, table)
    return table.contiguous(), n_pages


def _full_cache(c, seed, n_pages):
    """A cache whose every page holds keys and values."""
    Hkv, P, d = c["Hkv"], c["page"], c["d"]
    per = max(1, (1 << 27) // (Hkv * P * d))
    got = {}
    for name, key in (("k", True), ("v", False)):
        f = _outliers(seed, 2, Hkv * d).reshape(Hkv, 1, d) if key else 1.0
        g, parts = _gen(seed, 3 if key else 4), []
        for i in range(0, n_pages, per):
            x = torch.randn(min(per, n_pages - i), Hkv, P, d, generator=g, device="cuda") * f
            parts.append(_store(x, c["fmt"], c["group"], key))
        got[name] = torch.cat([p[0] for p in parts])
        got[name + "_stat"] = torch.cat([p[1] for p in parts]) if c["group"] else None
    return got


def _empty_cache(c, n_pages):
    Hkv, P, d = c["Hkv"], c["page"], c["d"]
    row, stat = _row_bytes(c)
    got = {}
    for name in ("k", "v"):
        got[name] = torch.zeros(n_pages, Hkv, P, row // 2 if c["fmt"] == "bf16" else row, device="cuda",
                                dtype=torch.bfloat16 if c["fmt"] == "bf16" else torch.uint8)
        got[name + "_stat"] = torch.zeros(n_pages, Hkv, stat // 4, P, 2, device="cuda",
                                          dtype=torch.bfloat16) if stat else None
    return got


def prepare(case, seed):
    c, kind, d = case, case["kind"], case["d"]
    f32, b16 = dict(device="cuda", dtype=torch.float32), dict(device="cuda", dtype=torch.bfloat16)
    if kind == "append":
        T, H, Hkv = c["n"] * c["tokens"], c["H"], c["Hkv"]
        end = c["start"] + c["tokens"]
        table, n_pages = _tables(c, seed, [end] * c["n"])
        seq, pos = _positions(c)
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        q = _normal(seed, 5, T, H * d).to(dt)
        kv = _normal(seed, 6, T, 2 * Hkv * d)
        kv[:, :Hkv * d] *= _outliers(seed, 2, Hkv * d)
        kv = kv.to(dt)
        k, v = kv[:, :Hkv * d], kv[:, Hkv * d:]
        if not c["stacked"]:
            k, v = k.contiguous(), v.contiguous()
        i = torch.arange(d // 2, device="cuda", dtype=torch.float64)
        ang = torch.arange(end, device="cuda", dtype=torch.float64)[:, None] * 1e4 ** (-2.0 * i / d)
        return dict(case=c, q=q, k=k, v=v, seq=seq, pos=pos, table=table, cache=_empty_cache(c, n_pages),
                    cs=torch.stack([ang.cos(), ang.sin()], -1).float().contiguous(),
                    q_out=torch.zeros(T, H * d, **b16),
                    start=torch.full((c["n"],), c["start"], device="cuda", dtype=torch.int32),
                    lens=torch.full((c["n"],), end, device="cuda", dtype=torch.int32),
                    K=torch.empty(Hkv, c["n"], c["tokens"], d, **b16),
                    V=torch.empty(Hkv, c["n"], c["tokens"], d, **b16))
    lens = _lens(c)
    table, n_pages = _tables(c, seed, lens)
    st = dict(case=c, table=table, lens=torch.tensor(lens, device="cuda", dtype=torch.int32),
              cache=_full_cache(c, seed, n_pages))
    if kind == "read":
        dt = f32 if c["out"] == "f32" else b16
        shape = (c["Hkv"], c["n"], c["L"], d)
        return dict(st, start=torch.full((c["n"],), c["start"], device="cuda", dtype=torch.int32),
                    K=torch.empty(shape, **dt), V=torch.empty(shape, **dt))
    return dict(st, q=_normal(seed, 5, c["n"], c["H"] * d).bfloat16(), scale=1.0 / d ** 0.5,
                O=torch.empty(c["n"], c["H"] * d, **b16), lse=torch.empty(c["n"], c["H"], **f32))


# ---------------------------------------------------------------------------
# run, the framework's calls
# ---------------------------------------------------------------------------
def _own_attn(s, ws):
    from paper_2506_03781_amd import uniquan as uq
    c, m = s["case"], s["cache"]
    uq.uniquan_attn_decode(c["n"], c["H"], c["Hkv"], c["d"], s["q"], s["lens"], s["table"], m["k"], m["v"], s["scale"],
                           s["O"], s["lse"], ws, fmt=KV[c["fmt"]], group=c["group"], page_len=c["page"],
                           k_stat=m["k_stat"], v_stat=m["v_stat"])


def _own_read(s, L):
    from paper_2506_03781_amd import uniquan as uq
    c, m = s["case"], s["cache"]
    uq.uniquan_kv_read(c["n"], c["Hkv"], c["d"], L, s["lens"], s["table"], m["k"], m["v"], s["K"], s["V"],
                       start=s["start"], fmt=KV[c["fmt"]], group=c["group"], page_len=c["page"], k_stat=m["k_stat"],
                       v_stat=m["v_stat"])


def _own_append(s):
    from paper_2506_03781_amd import uniquan as uq
    c, m = s["case"], s["cache"]
    uq.uniquan_kv_append(c["n"] * c["tokens"], c["H"], c["Hkv"], c["d"], s["q"], s["k"], s["v"], s["pos"], s["table"],
                         m["k"], m["v"], s["q_out"], seq=s["seq"], cs=s["cs"], fmt=KV[c["fmt"]], group=c["group"],
                         page_len=c["page"], k_stat=m["k_stat"], v_stat=m["v_stat"])
    if c["fmt"] != "bf16":
        _own_read(s, c["tokens"])


def _run_own(s):
    """A serving loop records its launches once and replays them."""
    from paper_2506_03781_amd import uniquan as uq
    c = s["case"]
    if "call" in s:
        s["call"]()
    elif c["kind"] == "attn":
        n = uq.uniquan_attn_decode_ws(c["n"], c["H"], c["Hkv"], c["d"], s["table"].shape[1], c["page"])
        s["ws"] = torch.empty(max(1, n), device="cuda")
        s["call"] = uq.record(_own_attn, s, s["ws"])
    elif c["kind"] == "append":
        s["call"] = uq.record(_own_append, s)
    else:
        s["call"] = uq.record(_own_read, s, c["L"])
    if c["kind"] == "attn":
        return dict(O=s["O"], lse=s["lse"])
    if c["kind"] == "read":
        return dict(K=s["K"], V=s["V"])
    if c["fmt"] == "bf16":
        return dict(q=s["q_out"], K=s["cache"]["k"], V=s["cache"]["v"])
    return dict(q=s["q_out"], K=s["K"], V=s["V"])


# ---------------------------------------------------------------------------
# run, plain torch
# ---------------------------------------------------------------------------
def _gathered(s, name):
    """fp32 values [n, Hkv, max_pages P, d] of every sequence's pages and which positions hold something."""
    c, m, t = s["case"], s["cache"], s["table"]
    has = (t >= 0) & (t < m[name].shape[0])
    idx = torch.where(has, t, 0).long()
    st = m[name + "_stat"]
    x = _values(m[name][idx], None if st is None else st[idx], c["fmt"], name == "k")
    x = x.transpose(1, 2).flatten(2, 3)
    at = torch.arange(x.shape[2], device="cuda")
    ok = has.repeat_interleave(c["page"], 1) & (at < s["lens"][:, None])
    return torch.where(ok[:, None, :, None], x, torch.zeros((), device="cuda")), ok


def _plain_attn(s):
    c = s["case"]
    q = s["q"].float().reshape(c["n"], c["Hkv"], -1, c["d"])
    K, ok = _gathered(s, "k")
    x = torch.matmul(q, K.transpose(2, 3)) * s["scale"]
    del K
    x = x.masked_fill(~ok[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    V, _ = _gathered(s, "v")
    o = torch.matmul(p, V) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)) * math.log2(math.e)
    return dict(O=o.reshape(c["n"], -1).bfloat16(), lse=lse.reshape(c["n"], -1))


def _plain_read(s, L):
    c, m, t, P = s["case"], s["cache"], s["table"], s["case"]["page"]
    at = s["start"][:, None].long() + torch.arange(L, device="cuda")
    ok = (at >= 0) & (at < s["lens"][:, None]) & (at < t.shape[1] * P)
    at = torch.where(ok, at, 0)
    page = t.gather(1, at // P).long()
    ok &= (page >= 0) & (page < m["k"].shape[0])
    page, r = torch.where(ok, page, 0), at % P
    out = []
    for name in ("k", "v"):
        st = m[name + "_stat"]
        x = _values(m[name][page, :, r].unsqueeze(3), None if st is None else st[page, :, :, r].unsqueeze(4), c["fmt"],
                    name == "k").squeeze(3)             # pages of one row: [n, L, Hkv, d]
        x = torch.where(ok[:, :, None, None], x, torch.zeros((), device="cuda"))
        out.append(x.permute(2, 0, 1, 3).to(s["K"].dtype).contiguous())
    return dict(K=out[0], V=out[1])


def _rotated(x, cs, heads, d):
    """x [T, heads d] with pairs (i, i + d / 2) of each head rotated by cs [T, d / 2, 2]."""
    a, b = x.float().unflatten(1, (heads, 2, d // 2)).unbind(2)
    co, si = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.stack([a * co - b * si, b * co + a * si], 2).flatten(2)


def _plain_append(s):
    c, m, d = s["case"], s["cache"], s["case"]["d"]
    rows = (s["pos"] >= 0).nonzero()[:, 0] if c["pad"] else torch.arange(s["pos"].shape[0], device="cuda")
    seq, pos = s["seq"][rows].long(), s["pos"][rows].long()
    page, slot = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    cs = s["cs"][pos]
    s["q_out"][rows] = _rotated(s["q"][rows], cs, c["H"], d).flatten(1).bfloat16()
    new = dict(k=_rotated(s["k"][rows], cs, c["Hkv"], d), v=s["v"][rows].float().unflatten(1, (c["Hkv"], d)))
    for name, x in new.items():
        row, st = _store(x[:, :, None], c["fmt"], c["group"], name == "k")    # pages of one row
        m[name][page, :, slot] = row[:, :, 0]
        if st is not None:
            m[name + "_stat"][page, :, :, slot] = st[:, :, :, 0]
    if c["fmt"] == "bf16":
        return dict(q=s["q_out"], K=m["k"], V=m["v"])
    return dict(q=s["q_out"], **_plain_read(s, c["tokens"]))


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "attn":
        return _plain_attn(state)
    return _plain_append(state) if kind == "append" else _plain_read(state, state["case"]["L"])


# ---------------------------------------------------------------------------
# work
# ---------------------------------------------------------------------------
def work(case):
    c, d = case, case["d"]
    row, stat = _row_bytes(c)
    if c["kind"] == "append":
        T = c["n"] * c["tokens"]
        T -= T // 8 if c["pad"] else 0
        w = 4 if c["dtype"] == "f32" else 2
        back = 0 if c["fmt"] == "bf16" else 2 * c["Hkv"] * (row + stat + 2 * d)
        each = (c["H"] + 2 * c["Hkv"]) * d * w + c["H"] * d * 2 + 2 * c["Hkv"] * (row + stat) + 4 * d + back
        return dict(bytes=T * each, flops=0)
    P, lens = c["page"], _lens(c)
    if c["kind"] == "read":
        held = sum(max(0, ln - c["start"]) for ln in lens)
        w = 4 if c["out"] == "f32" else 2
        return dict(bytes=2 * c["Hkv"] * (held * (row + stat) + c["n"] * c["L"] * d * w), flops=0)
    gone = sum(min(P, ln - j * P) for ln in lens for j in range(2, (ln + P - 1) // P, 4)) if c["holes"] else 0
    held = sum(lens) - gone
    return dict(bytes=2 * c["Hkv"] * held * (row + stat) + c["n"] * c["H"] * (4 * d + 4), flops=4 * held * c["H"] * d)


# ---------------------------------------------------------------------------
# exact: the same results in 64 bits from the definitions
# ---------------------------------------------------------------------------
def _places(c, key):
    """Byte and shift of every channel's code in a row."""
    d, bits = c["d"], 8 if c["fmt"] == "u8" else 4
    at, sh = [], []
    for ch in range(d):
        if key:
            j = ch % 8
            if bits == 4:
                j = j // 2 + 4 * (j % 2)
            p = (ch // 8) % 4 * (d // 4) + ch // 32 * 8 + j
        else:
            p = ch % 16 * (d // 16) + ch // 16
        at.append(p * bits // 8)
        sh.append(p * bits % 8)
    return torch.tensor(at, device="cuda"), torch.tensor(sh, device="cuda")


def _sequence64(s, name, i, first, last):
    """Values [Hkv, last - first, d] in 64 bits of sequence i's positions first..last - 1, and which hold something."""
    c, m = s["case"], s["cache"]
    P, d, pages = c["page"], c["d"], s["table"][i].tolist()
    p = torch.arange(first, last, device="cuda")
    page = torch.tensor([pages[j] for j in range(first // P, (last + P - 1) // P)], device="cuda")[p // P - first // P]
    ok = page >= 0
    page, r = page.clamp(min=0), p % P
    rows = m[name][page, :, r].transpose(0, 1)                     # [Hkv, positions, row]
    if c["fmt"] == "bf16":
        return rows.double(), ok
    at, sh = _places(c, name == "k")
    code = (rows[..., at].int() >> sh & TOP[c["fmt"]]).double()
    st = m[name + "_stat"][page, :, :, r].transpose(0, 1).double()  # [Hkv, positions, d / group, 2]
    grp = torch.arange(d, device="cuda") // c["group"]
    return st[..., 1][..., grp] + st[..., 0][..., grp] * code, ok


def exact(case, seed):
    c, d = case, case["d"]
    s = prepare(case, seed)
    if c["kind"] == "append":
        pos = s["pos"].long()
        ok = pos >= 0
        cs = s["cs"].double()[pos.clamp(min=0)][:, None]            # [T, 1, d / 2, 2]

        def turn(x):
            x = x.double().reshape(x.shape[0], -1, d)
            a, b = x[..., :d // 2], x[..., d // 2:]
            return torch.cat([a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]], -1)

        q = turn(s["q"]).flatten(1) * ok[:, None]
        if c["fmt"] != "bf16":
            return dict(q=q, K=None, V=None)  # codes follow from decisions in fp32
        out = dict(q=q)
        page = s["table"][s["seq"].long(), pos.clamp(min=0) // c["page"]].long()
        for name, x in (("K", turn(s["k"])), ("V", s["v"].double().reshape(-1, c["Hkv"], d))):
            buf = torch.zeros(s["cache"]["k"].shape, device="cuda", dtype=torch.float64)
            buf[page[ok], :, pos[ok] % c["page"]] = x[ok]
            out[name] = buf
        return out
    lens = s["lens"].tolist()
    if c["kind"] == "read":
        out = {}
        for name in ("k", "v"):
            buf = torch.zeros(s["K"].shape, device="cuda", dtype=torch.float64)
            for i, ln in enumerate(lens):
                if ln > c["start"]:
                    x, ok = _sequence64(s, name, i, c["start"], ln)
                    buf[:, i, :ln - c["start"]] = x * ok[None, :, None]
            out[name.upper()] = buf
        return out
    O = torch.zeros(c["n"], c["H"], d, device="cuda", dtype=torch.float64)
    lse = torch.full((c["n"], c["H"]), float("-inf"), device="cuda", dtype=torch.float64)
    for i, ln in enumerate(lens):
        if ln == 0:
            continue
        K, ok = _sequence64(s, "k", i, 0, ln)
        if not bool(ok.any()):
            continue
        x = s["q"][i].double().reshape(c["Hkv"], -1, d) @ K[:, ok].transpose(1, 2).contiguous() * (1.0 / d ** 0.5)
        del K
        V, _ = _sequence64(s, "v", i, 0, ln)
        O[i] = (torch.softmax(x, -1) @ V[:, ok]).reshape(c["H"], d)
        lse[i] = torch.logsumexp(x, -1).reshape(-1) / math.log(2.0)
    return dict(O=O.reshape(c["n"], -1), lse=lse)
