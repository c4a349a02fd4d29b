"""uniquan_sample against the plain reference (oracle.sample).

Tokens have to be equal: weights of the two differ by a unit at most, and a random border falls within V units of a
running sum (of at least 2^sh) with a probability of V^2 2^-sh, below 1e-4 for the largest row here and nothing to
be seen over a run of fixed seeds.  prob is a quotient of sums that agree to V 2^-sh, rounded to fp32: half a step of
2^-23 and as much again for the division in 64 bits and the weights."""
import numpy as np
import pytest
import torch

from oracle.sample import sample_row
from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu

NONE = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


def dev(a, dt=torch.float32):
    return None if a is None else torch.as_tensor(np.asarray(a)).to(dt).cuda()


def call(x, u, ws="own", **kw):
    """x: device rows; u and the settings host lists (None: not given)."""
    T, V = x.shape
    token, prob = torch.full((T,), -7, dtype=torch.int32, device="cuda"), torch.full((T,), -7.0, device="cuda")
    need = uq.uniquan_sample_ws(T, V)
    ws = torch.full((need,), float("nan"), device="cuda") if need else None
    opt = dict(temperature=dev(kw.get("temperature")), top_k=dev(kw.get("top_k"), torch.int32),
               top_p=dev(kw.get("top_p")), min_p=dev(kw.get("min_p")))
    uq.uniquan_sample(T, V, x, dev(u), token, prob=prob, ws=ws, **opt)
    torch.cuda.synchronize()
    return token.cpu().numpy(), prob.cpu().numpy()


def check(x, u, **kw):
    token, prob = call(x, u, **kw)
    rows = x.float().cpu().numpy()
    for r in range(len(rows)):
        one = {k: (NONE[k] if kw.get(k) is None else kw[k][r]) for k in NONE}
        want, p, _ = sample_row(rows[r], np.float32(u[r]), **one)
        assert token[r] == want, f"row {r} of {x.shape}, {one}, u {u[r]}: {token[r]}, expected {want}"
        assert abs(prob[r] - p) <= 2.0 ** -22 * p, f"row {r}: prob {prob[r]}, expected {p}"


def logits(rs, T, V, peaks=True):
    x = 2 * rs.standard_normal((T, V))
    if peaks:
        for r in range(T):
            x[r, rs.integers(0, V, 5)] += 6 + 3 * rs.standard_normal(5)
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 5, 63, 64, 65, 257, 1000, 4095, 4097, 8200, 20011, 50257])
def test_sizes(V, dtype):
    rs = np.random.default_rng(V)
    T = 9 if V < 10000 else 5
    x = dev(logits(rs, T, V), dtype)
    u = rs.random(T).astype(np.float32)
    t = rs.uniform(0.4, 1.5, T).astype(np.float32)
    k = rs.integers(1, 2 * V, T)
    p = rs.uniform(0.3, 1.05, T).astype(np.float32)
    lo = np.float32(10.0) ** rs.uniform(-6, -0.3, T).astype(np.float32)
    check(x, u)
    check(x, u, temperature=t)
    check(x, u, temperature=t, top_k=k)
    check(x, u, temperature=t, top_k=np.minimum(k, 50), top_p=p)
    check(x, u, temperature=t, top_p=p)
    check(x, u, min_p=lo)
    check(x, u, temperature=t, top_k=k, top_p=p, min_p=lo)


def test_a_large_row_and_wide_nuclei():
    """More tokens than are sorted at once, cut by value and by index."""
    rs = np.random.default_rng(3)
    V = 131075
    x = dev(logits(rs, 6, V))
    u = rs.random(6).astype(np.float32)
    check(x, u, top_k=[V // 2, 5000, 4096, 4097, 130000, 1], top_p=[0.99, 0.999, 0.5, 1.0, 0.9, 0.1])
    check(x, u, temperature=[3.0, 1.0, 10.0, 0.5, 100.0, 1e4], top_p=[0.99, 0.9, 0.95, 0.9999, 0.7, 0.3])
    check(x, u, temperature=[1e-4, 1e-30, 1e30, float("inf"), 1e-42, 2.0], top_k=[0, 7, 9000, 60000, 3, V])


@pytest.mark.parametrize("values", [1, 2, 7])
def test_many_equal_values(values):
    """A cut between equal values goes by the index."""
    rs = np.random.default_rng(values)
    V = 20000
    x = dev(rs.integers(0, values, (8, V)) * 0.25, torch.bfloat16)
    u = rs.random(8).astype(np.float32)
    check(x, u, top_k=[1, 4095, 4097, 7000, 12345, 19999, 20000, 300])
    check(x, u, top_p=[0.37, 0.1, 0.9, 0.99999, 1e-6, 0.5, 0.25, 0.75])
    check(x, u, top_k=[15000, 9000, 4097, 7000, 12345, 19999, 300, 1], top_p=[0.5, 0.9, 0.3, 0.99, 0.01, 0.7, 0.6, 0.5])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [3001, 20011])
def test_min_p_beside_the_others(V, dtype):
    """Few or many tokens left by min_p, alone, with top_p and with a large top_k; the last token kept too (u = 1)."""
    rs = np.random.default_rng(V)
    x = logits(rs, 12, V)
    x[3] = 0.5                                # all alike
    x[4, 100:] = -np.inf
    x[5, 7] = np.inf
    x[6, ::3] = np.nan
    x = dev(x, dtype)
    lo = np.array([0.3, 0.05, 1e-3, 0.5, 0.2, 0.1, 0.05, 1e-6, 1.0, 3e-2, 1e-30, 1e-45], np.float32)
    p = rs.uniform(0.2, 1.0, 12).astype(np.float32)
    k = rs.integers(513, V, 12)
    t = rs.uniform(0.4, 1.5, 12).astype(np.float32)
    t[10] = np.inf
    for u in (rs.random(12).astype(np.float32), np.ones(12, np.float32)):
        check(x, u, temperature=t, min_p=lo)
        check(x, u, temperature=t, min_p=lo, top_p=p)
        check(x, u, temperature=t, min_p=lo, top_k=k)
        check(x, u, temperature=t, min_p=lo, top_k=k, top_p=p)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("values", [1, 3])
def test_the_last_token_kept(values, dtype):
    """u = 1: the last one by index of those that stay, at cuts in every place of a chunk, in rows of every alignment."""
    rs = np.random.default_rng(values)
    V = 9001
    x = dev(rs.integers(0, values, (16, V)) * 0.25, dtype)
    k = 5000 + np.arange(16)
    check(x, np.ones(16, np.float32), top_k=k)
    check(x, np.ones(16, np.float32), top_k=k + 3000, top_p=[0.6] * 16)
    if values == 1:
        assert np.array_equal(call(x, np.ones(16), top_k=k)[0], k - 1)


def test_neighbouring_values_in_one_bin():
    """Values a few steps of fp32 apart: the cut is found among them."""
    rs = np.random.default_rng(11)
    V = 30000
    base = np.float32(1.0).view(np.int32)
    x = (base + rs.integers(0, 40, (4, V))).astype(np.int32).view(np.float32)
    x[2] = rs.integers(0, 3, V).astype(np.int32).view(np.float32) * np.where(rs.random(V) < 0.5, -1, 1)  # around 0
    x[3, :9000] = -x[3, :9000]
    u = rs.random(4).astype(np.float32)
    check(dev(x), u, top_k=[7001, 20000, 9001, 25000])
    check(dev(x), u, top_p=[0.3, 0.7, 0.5, 0.9])


def test_borders():
    x = np.zeros((8, 1000), np.float32)
    x[0, 3:] = -np.inf                       # three left
    x[1] = -np.inf                           # none
    x[2] = np.nan
    x[3, 17] = x[3, 400] = np.inf
    x[4, ::2] = np.nan
    x[5] = -3.4e38
    x[5, 999] = 3.4e38
    x[6, 0] = -np.inf
    x[6, 5] = -0.0
    x[7] = np.linspace(-40, 40, 1000)
    for u in (0.0, 0.3, 0.999999, 1.0, -1.0, 2.0):
        us = np.full(8, u, np.float32)
        check(dev(x), us)
        check(dev(x), us, top_k=[2] * 8, top_p=[0.5] * 8)
        check(dev(x), us, top_p=[0.0, -1.0, 0.1, 0.2, 0.5, 1.0, 0.9, 2.0], min_p=[1.0, 2.0, 0.5, 1.0, 1.0, 1e-3, 1.0, 0.5])
        check(dev(x), us, top_k=[0, -1, 1000, 1001, 1 << 30, 1, 999, 5])
        check(dev(x), us, temperature=[0.0, 0.0, -1.0, 0.0, 0.0, 0.0, 0.0, 0.0])
        check(dev(x, torch.bfloat16), us, top_k=[0, 0, 3, 3, 3, 3, 300, 3], min_p=[0.1] * 8)


def test_nan_settings():
    x = dev(logits(np.random.default_rng(0), 3, 500))
    nan = [float("nan")] * 3
    assert np.array_equal(call(x, nan)[0], call(x, [0.0] * 3)[0])
    assert np.array_equal(call(x, nan, temperature=nan)[0], x.argmax(1).cpu().numpy())
    u = [0.2, 0.5, 0.9]
    assert np.array_equal(call(x, u, top_p=nan, min_p=nan)[0], call(x, u)[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ld", [1003, 1024, 1501])
def test_rows_apart(ld, dtype):
    rs = np.random.default_rng(ld)
    wide = dev(np.full((7, ld), 100.0), dtype)
    wide[:, :1003] = dev(logits(rs, 7, 1003), dtype)
    u = rs.random(7).astype(np.float32)
    check(wide[:, :1003], u, top_k=[40] * 7)
    check(wide[:, :1003], u)


def test_no_rows_leave_everything():
    x = torch.empty(0, 50, device="cuda")
    token = torch.full((4,), -7, dtype=torch.int32, device="cuda")
    uq.uniquan_sample(0, 50, x, torch.empty(0, device="cuda"), token)
    assert (token == -7).all()


def test_shares_of_a_distribution():
    """Every token is drawn as often as its share of evenly spaced random numbers, to one draw."""
    p = np.array([0.5, 0.25, 0.125, 0.0625, 0.0625])
    T = 4096
    x = dev(np.log(p))[None].repeat(T, 1)
    token, prob = call(x, (np.arange(T) + 0.5) / T)
    got = np.bincount(token, minlength=5)
    assert np.abs(got - p * T).max() <= 1
    assert np.all(np.abs(prob - p[token]) <= 2.0 ** -20)


def test_captured_and_replayed():
    """A captured call reads what its buffers hold at each replay, with eager calls in between."""
    rs = np.random.default_rng(5)
    T, V = 6, 30011
    x = dev(logits(rs, T, V))
    u, k, p = dev(rs.random(T)), dev([50, 0, 9000, 1, 300, 20000], torch.int32), dev([0.9, 0.95, 0.99, 1.0, 0.5, 1.0])
    token, prob = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, device="cuda")
    need = uq.uniquan_sample_ws(T, V)
    ws = torch.empty(need, device="cuda") if need else None
    run = lambda: uq.uniquan_sample(T, V, x, u, token, prob=prob, top_k=k, top_p=p, ws=ws)  # noqa: E731
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i in range(4):
        x.copy_(dev(logits(rs, T, V)))
        u.copy_(dev(rs.random(T)))
        token.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        got = token.cpu().numpy()
        want, _ = call(x, u.cpu().numpy(), top_k=k.cpu().numpy(), top_p=p.cpu().numpy())
        assert np.array_equal(got, want), f"replay {i}"


def test_another_stream_and_repeated():
    rs = np.random.default_rng(8)
    x = dev(logits(rs, 40, 60000))
    u = rs.random(40).astype(np.float32)
    want = call(x, u, top_p=[0.98] * 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            got = call(x, u, top_p=[0.98] * 40)
            assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
