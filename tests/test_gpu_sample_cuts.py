"""uniquan_sample where its cuts change hands: at the end of a run of equal values that shares its bin with worse ones,
at the sizes where the kernel gathers, ranks, sorts or counts, and at the least top-p.  Bars as in test_gpu_sample."""
import numpy as np
import pytest
import torch

from oracle.sample import shift, weights
from paper_2506_03781_amd import uniquan as uq
from test_gpu_sample import call, check, dev

pytestmark = pytest.mark.gpu


def runs(rs, values, counts, V):
    """A row of V logits: counts[i] copies of values[i], the others of the last value, shuffled."""
    x = np.full(V, values[-1], np.float32)
    at = 0
    for v, n in zip(values, counts):
        x[at:at + n] = v
        at += n
    return rs.permutation(x)


def border_in_last(x, t, n, V=None):
    """The top-p that falls in the middle of the weight of the n-th token in order (x: the row of V, or its top k)."""
    w = sorted(weights(x, np.float32(t), shift(V or len(x))), reverse=True)
    return np.float32((sum(w[:n - 1]) + 0.5 * w[n - 1]) / sum(w))


def steps_below(x, n, dtype):
    """The value n steps of the type below x > 0."""
    if dtype == torch.float32:
        return (np.float32(x).view(np.int32) - np.int32(n)).view(np.float32)
    return (np.float32(x).view(np.int32) - np.int32(n << 16)).view(np.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("counts", [(2000,), (1500, 2000), (1025, 1030, 3000), (1024, 2000)])
def test_a_cut_at_the_end_of_a_run_of_equal_values(counts, dtype):
    """The first 1, 2 ... of the runs, and one token less and more, by top-k, by top-p and by both; values a step of the
    type apart (all in one bin, bf16 at a temperature of 200), alone and behind better tokens in bins before."""
    rs = np.random.default_rng(sum(counts))
    V, t, high = (10007, 1.0, 4.0) if dtype == torch.float32 else (10007, 200.0, 512.0)
    values = [steps_below(1.0, i, dtype) for i in range(len(counts) + 1)]
    x, k, p, both = [], [], [], []
    for better in (0, 30):
        for end in better + np.cumsum(counts):
            for n in (int(end) - 1, int(end), int(end) + 1):
                row = runs(rs, [high, *values], [better, *counts], V)
                more = min(V, n + 700)
                x.append(row)
                k.append(n)
                p.append(border_in_last(row, t, n))
                both.append((more, border_in_last(-np.sort(-row)[:more], t, n, V)))
    T = len(x)
    xs = dev(np.stack(x), dtype)
    for u in (np.ones(T, np.float32), rs.random(T).astype(np.float32)):
        check(xs, u, temperature=[t] * T, top_k=k)
        check(xs, u, temperature=[t] * T, top_p=p)
        check(xs, u, temperature=[t] * T, top_k=[b[0] for b in both], top_p=[b[1] for b in both])
        check(xs, u, temperature=[t] * T, top_k=k, min_p=[0.5] * T)


def test_a_cut_at_the_end_of_a_run_of_infinities():
    """Of 3000 logits of +infinity the first 2999, all, and no more than all."""
    rs = np.random.default_rng(1)
    x = np.stack([runs(rs, [np.float32(np.inf), np.float32(1.0)], [3000], 9000) for _ in range(6)])
    for u in (1.0, 0.5):
        check(dev(x), np.full(6, u, np.float32), top_k=[2999, 3000, 3001, 0, 0, 3000], top_p=[1.0, 1.0, 1.0, 0.9999, 0.5, 0.9])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 31, 32, 33, 127, 128, 129, 511, 512, 513, 1023, 1024, 1025, 1026])
def test_as_many_tokens_as_change_the_way(n, dtype):
    """n tokens stand out of 8011, side by side or scattered: by top-k (512 is the most that the lanes' best tokens are
    asked for), and gathered by top-p and by min-p as a list of n (of up to 1024, by min-p of those of up to half the
    lanes; up to 128 are ranked, up to 32 by 32 threads each)."""
    rs = np.random.default_rng(n)
    V = 8011
    x = rs.uniform(-26, -25, (6, V))
    for r in range(6):
        at = rs.permutation(V)[:n] if r < 3 else int(rs.integers(0, V - n)) + np.arange(n)
        x[r, at] = rs.uniform(0.0, 1.0, n) if r % 3 == 1 else rs.uniform(0.4, 0.5, n)
    xs = dev(x, dtype)
    u = rs.random(6).astype(np.float32)
    u[[0, 1, 4, 5]] = 1.0
    check(xs, u, top_k=[n] * 6)
    check(xs, u, top_k=[n + 1, max(1, n - 1)] * 3, top_p=[0.9] * 6)
    check(xs, u, top_p=[0.9999995] * 6)
    check(xs, u, top_p=[0.9999995] * 6, min_p=[1e-3] * 6)
    check(xs, u, min_p=[1e-3] * 6)
    check(xs, u, top_k=[5000] * 6, min_p=[1e-3] * 6)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_least_top_p(dtype):
    """Any top-p above 0 keeps the first token: numbers below 2^-64, with subnormal ones, alone and beside the others."""
    rs = np.random.default_rng(2)
    p = np.array([1e-20, 1e-45, 2.0 ** -64, 2.0 ** -65, 5.5e-20, 1e-38, 1e-12, 2.0 ** -63], np.float32)
    for V in (5, 300, 8011):
        x = rs.standard_normal((8, V))
        x[4:] = 0.25                              # all alike: the first by index
        xs = dev(x, dtype)
        for u in (np.zeros(8, np.float32), np.ones(8, np.float32), rs.random(8).astype(np.float32)):
            check(xs, u, top_p=p)
            check(xs, u, top_p=p, top_k=[50, 1, 3, 2, 50, 1, 600, 2])
            check(xs, u, top_p=p, top_k=[5000] * 8, min_p=[0.1] * 8)
            check(xs, u, top_p=p, min_p=[0.1, 1.0, 1e-3, 0.5] * 2)
            check(xs, u, top_p=p, temperature=[100.0] * 8)


def test_more_rows_than_a_dimension_of_the_grid_takes():
    """2^22 rows and five (1024 threads each: 2^32 and more), equal to the rows in two calls, greedy ones to argmax."""
    g = torch.Generator(device="cuda").manual_seed(3)
    T, V, cut = (1 << 22) + 5, 3, 1 << 21
    x, u = torch.randn(T, V, generator=g, device="cuda"), torch.rand(T, generator=g, device="cuda")
    t = torch.ones(T, device="cuda")
    t[::3] = 0.0
    token, prob = torch.full((T + 9,), -7, dtype=torch.int32, device="cuda"), torch.full((T + 9,), -7.0, device="cuda")
    uq.uniquan_sample(T, V, x, u, token, prob=prob, temperature=t)
    t2, p2 = torch.empty(T, dtype=torch.int32, device="cuda"), torch.empty(T, device="cuda")
    for a, b in ((0, cut), (cut, T)):
        uq.uniquan_sample(b - a, V, x[a:b], u[a:b], t2[a:b], prob=p2[a:b], temperature=t[a:b].contiguous())
    torch.cuda.synchronize()
    assert (token[T:] == -7).all() and (prob[T:] == -7.0).all()
    assert torch.equal(token[:T], t2) and torch.equal(prob[:T], p2)
    assert torch.equal(token[:T][::3].long(), x[::3].argmax(1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1 << 22, (1 << 22) - 3, 1 << 20])
def test_the_largest_rows(V, dtype):
    """The plain reference's steps on whole arrays: its integers fit 64 bits (V 2^sh is 2^62 at most)."""
    g = torch.Generator(device="cuda").manual_seed(V % 100)
    x = (2 * torch.randn(V, generator=g, device="cuda")).to(dtype)
    row = x.float().cpu().numpy()
    sh = shift(V)
    w = np.rint(np.exp(row.astype(np.longdouble) - np.longdouble(row.max())) * np.longdouble(2.0) ** sh).astype(np.int64)
    order = np.lexsort((np.arange(V), -row))
    before = np.cumsum(w[order]) - w[order]
    total = int(w.sum())
    k = [0, 0, 1000, 600000, 0, V - 1]
    p = np.array([1.0, 0.9, 0.8, 0.95, 0.999, 1.0], np.float32)
    lo = np.array([0, 0, 0, 0, 1e-3, 1e-5], np.float32)
    u = np.array([0.3, 0.8, 0.999, 0.5, 1.0, 0.7], np.float32)
    token, prob = call(x[None].repeat(6, 1), u, top_k=k, top_p=p, min_p=lo)
    for r in range(6):
        first = order[:k[r]] if k[r] else order
        if p[r] < 1:
            mass = int(w[first].sum())
            border = -(-int(np.float64(p[r]) * 2.0 ** 64) * mass >> 64)  # ceil
            first = first[before[:len(first)] < border]
        if lo[r] > 0:
            first = first[w[first] >= np.ceil(np.float64(lo[r]) * 2.0 ** sh)]
        kept = np.sort(first)
        upto = np.cumsum(w[kept])
        mass = int(upto[-1])
        at = mass - 1 if u[r] >= 1 else int(np.float64(u[r]) * 2.0 ** 64) * mass >> 64
        want = kept[np.searchsorted(upto, at, side="right")]
        assert token[r] == want, f"row {r}: {token[r]}, expected {want}"
        assert abs(prob[r] - w[want] / mass) <= 2.0 ** -22 * w[want] / mass
    assert total <= 1 << 62
