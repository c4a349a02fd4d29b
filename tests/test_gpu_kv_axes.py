"""uniquan_kv_append_axes: rows rotated at positions of their own, on several axes.

The rotation in fp32 without contraction is the same in numpy, so the cache and the queries have to equal, bit for
bit, what uniquan_kv_append without a table stores of rows that numpy rotated; the rotation itself against 64 bits:
two products and a sum, each rounded once, within 3 2^-24 (|x1| + |x2|)."""
import numpy as np
import pytest
import torch

import kv_cases as C
from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu
F32 = np.float32


def rotated(x, rot, axis, cs, heads, d, bits=F32):
    """x [T, heads d] with pair i of row t turned by cs[rot[t, axis[i]], i]; other axes: not turned."""
    T, n_axes = rot.shape
    y = x.astype(bits).reshape(T, heads, 2, d // 2)
    a, b = y[:, :, 0].copy(), y[:, :, 1].copy()
    for i in range(d // 2):
        if 0 <= axis[i] < n_axes:
            c, s = (cs[rot[:, axis[i]], i, e].astype(bits)[:, None] for e in range(2))
            y[:, :, 0, i] = a[..., i] * c - b[..., i] * s
            y[:, :, 1, i] = b[..., i] * c + a[..., i] * s
    return y.reshape(T, heads * d)


def empty(rs, n, H_kv, d, P, fmt, group, per=5):
    n_pages = n * per + 2
    row = dict(bf16=d, u8=d, u4=d // 2)[fmt]
    dt = torch.bfloat16 if fmt == "bf16" else torch.uint8
    g = 0 if fmt == "bf16" else C.group_of(group, d)
    m = dict(table=C.dev(rs.permutation(n_pages)[:n * per].reshape(n, per).astype(np.int32)),
             k_cache=torch.full((n_pages, H_kv, P, row), 77, dtype=dt, device="cuda"),
             v_cache=torch.full((n_pages, H_kv, P, row), 77, dtype=dt, device="cuda"), k_stat=None, v_stat=None,
             fmt=C.FMT[fmt], group=g, page_len=P)
    if g:
        for s in ("k_stat", "v_stat"):
            m[s] = torch.full((n_pages, H_kv, d // g, P, 2), 5.0, dtype=torch.bfloat16, device="cuda")
    return m


def copy_of(m):
    return {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in m.items()}


def same(a, b):
    for k in ("k_cache", "v_cache", "k_stat", "v_stat"):
        if a[k] is not None:
            assert np.array_equal(C.host_bits(a[k]), C.host_bits(b[k])), k


def axes_call(m, T, H, H_kv, d, q, k, v, pos, rot, axis, cs, q_out, seq):
    uq.uniquan_kv_append_axes(T, H, H_kv, d, q, k, v, pos, rot, axis, cs, m["table"], m["k_cache"], m["v_cache"],
                              q_out=q_out, seq=seq, fmt=m["fmt"], group=m["group"], page_len=m["page_len"],
                              k_stat=m["k_stat"], v_stat=m["v_stat"])


def plain_call(m, T, H, H_kv, d, q, k, v, pos, q_out, seq, cs=None):
    uq.uniquan_kv_append(T, H, H_kv, d, q, k, v, pos, m["table"], m["k_cache"], m["v_cache"], q_out=q_out, seq=seq,
                         cs=cs, fmt=m["fmt"], group=m["group"], page_len=m["page_len"], k_stat=m["k_stat"],
                         v_stat=m["v_stat"])


def axis_of(kind, d, n_axes):
    i = np.arange(d // 2)
    if kind == "runs":
        return np.minimum(i * n_axes // (d // 2), n_axes - 1)
    if kind == "mixed":
        return i % n_axes
    return np.where(i % 3 == 1, -1, np.where(i % 5 == 2, n_axes, i % n_axes))  # some pairs on no axis


@pytest.mark.parametrize("fmt,group", C.FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_axes,kind", [(1, "runs"), (3, "runs"), (3, "mixed"), (8, "mixed"), (2, "part")])
def test_rows_at_positions_of_their_own(fmt, group, d, n_axes, kind):
    rs = np.random.default_rng(d + n_axes)
    n, H_kv, H, P, T = 3, 2, 6, 16, 31
    n_cs = 40
    cs = C.cos_sin(n_cs, d)
    rot = rs.integers(0, n_cs, (T, n_axes))
    axis = axis_of(kind, d, n_axes)
    seq, pos = np.arange(T) % n, np.arange(T) // n * 7 % 80       # places past the table's length too
    q, k, v = (rs.standard_normal((T, h * d)).astype(F32) for h in (H, H_kv, H_kv))
    rq, rk = rotated(q, rot, axis, cs, H, d), rotated(k, rot, axis, cs, H_kv, d)
    wide = rotated(q, rot, axis, cs, H, d, np.float64)
    size = np.abs(q).reshape(T, H, 2, -1).sum(2, keepdims=True).repeat(2, 2).reshape(T, -1)
    assert np.all(np.abs(rq - wide) <= 3 * 2.0 ** -24 * size)
    m = empty(rs, n, H_kv, d, P, fmt, group)
    want = copy_of(m)
    i32 = lambda a: C.dev(np.asarray(a).astype(np.int32))  # noqa: E731
    out, ref = (torch.full((T, H * d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    axes_call(m, T, H, H_kv, d, C.dev(q), C.dev(k), C.dev(v), i32(pos), i32(rot), i32(axis), C.dev(cs), out, i32(seq))
    plain_call(want, T, H, H_kv, d, C.dev(rq), C.dev(rk), C.dev(v), i32(pos), ref, i32(seq))
    same(m, want)
    assert np.array_equal(C.host_bits(out), C.host_bits(ref))


@pytest.mark.parametrize("T", [1, 5, 1700])
def test_one_axis_at_the_places_is_the_plain_call(T):
    rs = np.random.default_rng(T)
    n, H_kv, H, d, P = T, 4, 8, 128, 16
    cs = C.dev(C.cos_sin(80, d))
    m = empty(rs, n, H_kv, d, P, "u8", 32)
    want = copy_of(m)
    q, k, v = (C.dev(rs.standard_normal((T, h * d)).astype(F32)).bfloat16() for h in (H, H_kv, H_kv))
    pos = C.dev(rs.integers(0, 80, T).astype(np.int32))
    out, ref = (torch.zeros(T, H * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    axes_call(m, T, H, H_kv, d, q, k, v, pos, pos[:, None].contiguous(), torch.zeros(64, dtype=torch.int32, device="cuda"),
              cs, out, None)
    plain_call(want, T, H, H_kv, d, q, k, v, pos, ref, None, cs=cs)
    same(m, want)
    assert np.array_equal(C.host_bits(out), C.host_bits(ref))


def test_padding_leaves_everything():
    """Rows with a place, a sequence or any rotary position out of range; infinities beside a pair on no axis."""
    rs = np.random.default_rng(1)
    d, H_kv, P = 64, 2, 16
    cs = C.cos_sin(10, d)
    axis = np.zeros(d // 2, int)
    axis[3] = 5                                   # on no axis
    rot = np.array([[0, 0], [-1, 0], [0, 10], [0, 0], [0, 0], [0, 0], [3, 9], [1 << 30, 0], [0, -(1 << 31)]])
    pos = np.array([0, 1, 2, -1, 80, 3, 4, 5, 6])
    seq = np.array([0, 0, 0, 0, 0, 1, 0, 0, 0])
    T = len(pos)
    q, k, v = (rs.standard_normal((T, H_kv * d)).astype(F32) for _ in range(3))
    k[0, 3] = np.inf                              # its partner stays finite
    m = empty(rs, 1, H_kv, d, P, "bf16", 0)
    want = copy_of(m)
    i32 = lambda a: C.dev(np.asarray(a).astype(np.int32))  # noqa: E731
    out = torch.full((T, H_kv * d), 9.0, dtype=torch.bfloat16, device="cuda")
    axes_call(m, T, H_kv, H_kv, d, C.dev(q), C.dev(k), C.dev(v), i32(pos), i32(rot), i32(axis), C.dev(cs), out, i32(seq))
    good = [0, 6]
    ref = torch.full((2, H_kv * d), 9.0, dtype=torch.bfloat16, device="cuda")
    plain_call(want, 2, H_kv, H_kv, d, C.dev(rotated(q, rot.clip(0, 9), axis, cs, H_kv, d)[good]),
               C.dev(rotated(k, rot.clip(0, 9), axis, cs, H_kv, d)[good]), C.dev(v[good]), i32(pos[good]), ref, i32(seq[good]))
    same(m, want)
    got = out.float().cpu().numpy()
    assert np.array_equal(got[good], ref.float().cpu().numpy())
    assert np.all(got[[i for i in range(T) if i not in good]] == 9.0)


def test_without_queries_and_captured():
    rs = np.random.default_rng(2)
    d, H_kv, P, T = 128, 2, 32, 6
    m = empty(rs, T, H_kv, d, P, "u4", 32)
    cs = C.dev(C.cos_sin(50, d))
    kv = C.dev(rs.standard_normal((T, 2 * H_kv * d)).astype(F32))
    k, v = kv[:, :H_kv * d], kv[:, H_kv * d:]
    pos, rot = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((T,), (T, 2)))
    axis = C.dev((np.arange(64) % 2).astype(np.int32))
    run = lambda c: axes_call(c, T, H_kv, H_kv, d, None, k, v, pos, rot, axis, cs, None, None)  # noqa: E731
    run(copy_of(m))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(m)
    for i in range(3):
        pos += 7
        rot[:, 0] += 3
        rot[:, 1] += 11
        want = copy_of(m)
        g.replay()
        run(want)
        torch.cuda.synchronize()
        same(m, want)
