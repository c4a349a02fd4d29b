"""The paged key/value cache on the device (uniquan_kv_append, uniquan_kv_read)
against oracle/kv_cache.py: rotated values, codes, scales and offsets bit for
bit, and what no row names left as it was."""
import numpy as np
import pytest
import torch

import oracle.kv_cache as KV
from kv_cases import FORMS, cos_sin, dev, filled, group_of, host_bits, on_device, poison, rounded, same_cache, tables
from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu
F32 = np.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    uq.lib()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def to_dtype(x, dt):
    """Device tensor of host fp32 values and the values it holds."""
    t = dev(x, torch.float32).to(dt)
    return t, t.float().cpu().numpy()


def run_append(c, q, k, v, pos, seq, cs, dt, stacked=False):
    """Append on the device and on the host; both caches and q rows compared."""
    T, H, d = q.shape
    tq, q = to_dtype(q.reshape(T, -1), dt)
    if stacked:
        both, x = to_dtype(np.concatenate([k.reshape(T, -1), v.reshape(T, -1)], 1), dt)
        n = k.shape[1] * d
        tk, tv, k, v = both[:, :n], both[:, n:], x[:, :n], x[:, n:]
    else:
        tk, k = to_dtype(k.reshape(T, -1), dt)
        tv, v = to_dtype(v.reshape(T, -1), dt)
    q_out = np.full((T, H * d), 0x7FC1, np.uint16)
    tq_out, m = dev(q_out), on_device(c)
    uq.uniquan_kv_append(T, H, c.n_kv, d, tq, tk, tv, dev(np.asarray(pos, np.int32)), q_out=tq_out,
                         seq=None if seq is None else dev(np.asarray(seq, np.int32)),
                         cs=None if cs is None else dev(cs), **m)
    torch.cuda.synchronize()
    c.append(k.reshape(T, c.n_kv, d), v.reshape(T, c.n_kv, d), pos, q.reshape(T, H, d), q_out, seq, cs)
    same_cache(m, c)
    assert np.array_equal(host_bits(tq_out), q_out)
    return m


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d,n_kv,grp,P", [(128, 2, 4, 16), (64, 3, 1, 32), (128, 1, 7, 64), (64, 1, 2, 1024)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_append_prompts(fmt, group, d, n_kv, grp, P, dt):
    """Parts of prompts of unequal lengths, from positions inside pages, rows in a drawn order."""
    rs = np.random.default_rng(d + n_kv + P)
    first, count = [0, 13, 31, 5], [37, 1, 20, 0]
    t, n_pages = tables(rs, [a + b for a, b in zip(first, count)], P)
    c = KV.Cache(n_pages, n_kv, d, P, fmt, group_of(group, d) if fmt != "bf16" else 0, t)
    poison(c)
    rows = [(s, p) for s in range(4) for p in range(first[s], first[s] + count[s])]
    rows = [rows[i] for i in rs.permutation(len(rows))]
    seq, pos = [r[0] for r in rows], [r[1] for r in rows]
    T = len(rows)
    q, k, v = (rs.standard_normal((T, n, d)).astype(F32) for n in (n_kv * grp, n_kv, n_kv))
    k[:, :, 3] *= 20
    run_append(c, q, k, v, pos, seq, cos_sin(60, d), dt, stacked=P == 32)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d,n_kv,grp", [(64, 18, 4), (128, 17, 1)])
def test_append_many_rows_of_many_heads(fmt, group, d, n_kv, grp):
    """A prompt whose rows have a workgroup each, several tiles of heads to a row."""
    rs = np.random.default_rng(n_kv)
    T, P = 1601, 32
    t, n_pages = tables(rs, [T], P)
    c = KV.Cache(n_pages, n_kv, d, P, fmt, group_of(group, d) if fmt != "bf16" else 0, t)
    poison(c)
    q, k, v = (rs.standard_normal((T, n, d)).astype(F32) for n in (n_kv * grp, n_kv, n_kv))
    pos = np.arange(T)
    pos[[3, 900]] = -1
    run_append(c, q, k, v, pos, np.zeros(T, np.int32), cos_sin(T, d), torch.bfloat16)


@pytest.mark.parametrize("fmt,group", FORMS)
def test_append_rows_that_go_nowhere(fmt, group):
    """Padding, positions behind the table or the rotary table, sequences and pages that are none: nothing is written
    for them and their queries stay, except that a row without a page still gets its query."""
    rs = np.random.default_rng(7)
    table = [[4, -1, 99], [0, 5, 1], [-7, 2, 3]]
    c = KV.Cache(6, 2, 128, 16, fmt, group_of(group, 128) if fmt != "bf16" else 0, table)
    poison(c)
    seq = [0, 0, 0, 0, 1, 1, 1, 2, 2, 3, -1, 1]
    pos = [0, 17, 33, -1, 47, 48, 40, 3, 18, 2, 2, -(1 << 31)]
    q, k, v = (rs.standard_normal((12, n, 128)).astype(F32) for n in (4, 2, 2))
    run_append(c, q, k, v, pos, seq, cos_sin(41, 128), torch.float32)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_append_edge_values(fmt, group, d):
    """Constant groups, zeros, tiny, huge and non-finite values, negative offsets, no rotation."""
    rs = np.random.default_rng(8)
    T = 14
    x = rs.standard_normal((T, 1, d)).astype(F32)
    x[0] = 0
    x[1] = 3.3
    x[2] = -7.0001
    x[3] *= 1e-38
    x[4] *= 1e-42
    x[5] *= 1e37
    x[6, 0, 5] = np.inf
    x[7, 0, d - 1] = -np.inf
    x[8, 0, 40] = np.nan
    x[9, 0, 0], x[9, 0, 1] = 3e38, -3e38
    x[10] = 1000 + 1e-3 * x[10]
    x[11] = np.abs(x[11])
    x[12] = -np.abs(x[12])
    x[13] = -0.0
    t, n_pages = tables(rs, [T], 16)
    c = KV.Cache(n_pages, 1, d, 16, fmt, group_of(group, d) if fmt != "bf16" else 0, t)
    poison(c)
    if fmt == "bf16":  # NaN bits of a bf16 store are any NaN
        x[8, 0, 40] = 1
    run_append(c, x, x, x[::-1].copy(), list(range(T)), [0] * T, None, torch.float32)


def test_append_without_queries_and_strided_rows():
    rs = np.random.default_rng(9)
    t, n_pages = tables(rs, [9, 9, 9], 16)
    c = KV.Cache(n_pages, 2, 64, 16, "u4", 32, t)
    k, v = (rs.standard_normal((3, 2, 64)).astype(F32) for _ in range(2))
    wide = torch.zeros(3, 4, 128, device="cuda")
    wide[:, 1], wide[:, 3] = dev(k).reshape(3, 128), dev(v).reshape(3, 128)
    m = on_device(c)
    flat = wide.reshape(3, 512)
    uq.uniquan_kv_append(3, 2, 2, 64, None, flat[:, 128:256], flat[:, 384:], dev(np.array([8, 0, 3], np.int32)), **m)
    torch.cuda.synchronize()
    c.append(k, v, [8, 0, 3])
    same_cache(m, c)


def test_append_nothing():
    c = KV.Cache(2, 1, 64, 16, "u8", 32, [[0, 1]])
    m = on_device(c)
    e = torch.empty(0, 64, device="cuda")
    uq.uniquan_kv_append(0, 1, 1, 64, None, e, e, torch.empty(0, dtype=torch.int32, device="cuda"), **m)
    torch.cuda.synchronize()
    same_cache(m, c)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d,n_kv,P", [(128, 3, 16), (64, 2, 64)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_read(fmt, group, d, n_kv, P, dt):
    """Ranges that start before, inside and behind sequences, over missing pages; both arrays or one."""
    rs = np.random.default_rng(d + P)
    lens = [70, 0, 1, 33, 200]
    c = filled(rs, lens, n_kv, d, P, fmt, group)
    c.table[4, 1] = -1
    c.table[0, 0] = c.n_pages
    m = on_device(c)
    given = [70, -4, 1, 33, 10 ** 6]
    for L, start in ((40, None), (1, [69, 0, 0, 33, 199]), (75, [-3, 5, 0, 20, 150])):
        K, V = (torch.full((n_kv, 5, L, d), float("nan"), device="cuda", dtype=dt) for _ in range(2))
        kw = dict(start=None if start is None else dev(np.array(start, np.int32)), **m)
        lens_d = dev(np.array(given, np.int32))
        uq.uniquan_kv_read(5, n_kv, d, L, lens_d, K=K, V=V, **kw)
        torch.cuda.synchronize()
        rk, rv = c.read([70, 0, 1, 33, c.table.shape[1] * P], L, start)
        for got, ref in ((K, rk), (V, rv)):
            ref = ref if dt == torch.float32 else KV.bf16(ref)
            g = host_bits(got)
            nan = np.isnan(ref) if dt == torch.float32 else np.isnan(KV.from_bf16(ref))
            assert np.array_equal(g[~nan], ref[~nan]) and bool(torch.isnan(got).cpu().numpy()[nan].all())
        alone = torch.full_like(V, float("nan"))
        uq.uniquan_kv_read(5, n_kv, d, L, lens_d, K=None, V=alone, **kw)
        assert np.array_equal(host_bits(alone), host_bits(V), equal_nan=dt == torch.float32)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes a side: rows at its far end are written and come back."""
    d, n_kv, P = 128, 8, 256
    n_pages = (1 << 32) // (n_kv * P * d * 2) + 3
    far = n_pages - 1
    k_cache, v_cache = (torch.zeros(n_pages, n_kv, P, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[0, far], [far - 1, 1]], dtype=torch.int32, device="cuda")
    m = dict(table=table, k_cache=k_cache, v_cache=v_cache, page_len=P)
    rs = np.random.default_rng(3)
    k, v = (dev(rounded(rs, 2, n_kv * d)) for _ in range(2))
    uq.uniquan_kv_append(2, n_kv, n_kv, d, None, k, v, dev(np.array([P + 255, 3], np.int32)), **m)
    K, V = (torch.empty(n_kv, 2, 1, d, device="cuda") for _ in range(2))
    uq.uniquan_kv_read(2, n_kv, d, 1, dev(np.array([2 * P, P], np.int32)), K=K, V=V,
                       start=dev(np.array([P + 255, 3], np.int32)), **m)
    torch.cuda.synchronize()
    assert torch.equal(K[:, :, 0].transpose(0, 1).reshape(2, -1), k)
    assert torch.equal(V[:, :, 0].transpose(0, 1).reshape(2, -1), v)
    assert torch.equal(k_cache[far, :, 255].float().reshape(-1), k[0])


def test_append_millions_of_rows():
    """More rows than a grid dimension's workgroups: the first and the last one stored, the rest padding."""
    T, d, P = (1 << 20) + 77, 64, 16
    rs = np.random.default_rng(19)
    c = KV.Cache(2, 1, d, P, "bf16", 0, [[1]])
    poison(c)
    m = on_device(c)
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    at = [0, 1 << 20, T - 1]
    rows = rounded(rs, 3, 1, d)
    x[at] = dev(rows[:, 0]).bfloat16()
    pos = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    pos[at] = torch.tensor([2, 3, 4], dtype=torch.int32, device="cuda")
    uq.uniquan_kv_append(T, 1, 1, d, None, x, x, pos, seq=torch.zeros_like(pos), **m)
    torch.cuda.synchronize()
    c.append(rows, rows, [2, 3, 4], seq=[0, 0, 0])
    same_cache(m, c)


def test_read_millions_of_sequences():
    """More sequences than a grid dimension's workgroups take: the first and the last ones hold something."""
    n, d, P = (1 << 21) + 9, 64, 16
    rs = np.random.default_rng(20)
    some = [0, 1 << 20, 1 << 21, n - 1]
    c = filled(rs, [16] * 4, 1, d, P, "u8", 32)
    m = on_device(c)
    table = torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
    table[some] = m["table"]
    m["table"] = table
    lens, start = (torch.full((n,), x, dtype=torch.int32, device="cuda") for x in (16, 7))
    K, V = (torch.full((1, n, 1, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    uq.uniquan_kv_read(n, 1, d, 1, lens, K=K, V=V, start=start, **m)
    torch.cuda.synchronize()
    for got, want in zip((K, V), c.read([16] * 4, 1, [7] * 4)):
        assert np.array_equal(host_bits(got[0, some, 0]), KV.bf16(want[0, :, 0]))
        assert int((got != 0).any(-1).sum()) == 4 and not bool(got.isnan().any())
