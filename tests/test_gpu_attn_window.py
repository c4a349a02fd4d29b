"""uniquan_attn_window_fwd / _bwd against the formulas in 64 bits and against differences.

Bars, element by element, from the roundings alone (u = 2^-24; bf16 rounds by 2^-8 of a value at most):
  scores   d products and sums in fp32, scale, exponent: dx = (d + 16) u max scale sum |q||k| of the row; weights are
           then off by e^(2 dx) - 1 (numerator and log-sum-exp), and 2^-20 for the exponential and the logarithm
  P        2^-8 more in the products with V and dO; O is stored in bf16, 2^-8
  dP       (d + 4) u sum |dO||V|;  delta = sum P dP: the errors of both, and (n + 4) u sum P |dP|
  dS       weights' error of P |dP - delta|, P times the errors of dP and delta, 2^-8 for its rounding
  sums over n terms in fp32: (n + 4) u of the terms' absolute sum; outputs in bf16 2^-8; a rotated pair carries the
  bars of both its halves, and 2^-22 for the table and its products."""
import math

import numpy as np
import pytest
import torch

from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu
D, U, H8 = 128, 2.0 ** -24, 2.0 ** -8


def seen_of(L, window, sinks):
    i = torch.arange(L, device="cuda")
    gap = i[:, None] - i
    return (gap >= 0) & ((gap < window) | (i < sinks))


def cos_sin(L):
    cs = torch.empty(L, D // 2, 2, device="cuda")
    uq.uniquan_rope_table(L, D, cs)
    return cs


class Case:
    """Drawn operands; n sequences, H query heads on Hkv."""

    def __init__(self, L, window, sinks, n=1, H=2, Hkv=2, seed=0, size=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed + 31 * L + window)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
        self.L, self.window, self.sinks, self.n, self.H, self.Hkv = L, window, sinks, n, H, Hkv
        self.Q, self.K, self.V = r(H * n, L, D) * size, r(Hkv * n, L, D), r(Hkv * n, L, D)
        self.dO = r(H * n, L, D)                       # head-major
        self.scale = D ** -0.5

    def token(self, x, heads):
        """Head-major [heads n, L, d] (grouped slots for query heads) as token-major rows."""
        G = heads // self.Hkv
        return x.reshape(G, self.Hkv, self.n, self.L, D).permute(2, 3, 1, 0, 4).reshape(self.n * self.L, heads * D)

    def run(self, tok):
        L, n, H, Hkv, bw = self.L, self.n, self.H, self.Hkv, (self.H * self.n, self.Hkv * self.n)
        e = lambda *s, dt=torch.float32: torch.full((math.prod(s) + 64,), 7.0, dtype=dt, device="cuda")  # noqa: E731
        b16 = torch.bfloat16
        O, lse, delta = e(bw[0], L, D, dt=b16), e(bw[0], L), e(bw[0], L)
        one = tok and H == Hkv
        dQ = e(bw[0], L, D, dt=b16 if tok else torch.float32)
        dK, dV = (e(bw[0], L, D, dt=b16 if one else torch.float32) for _ in range(2))
        how = dict(tok_seqs=n, group=H // Hkv) if tok else {}
        nq = bw[0] * L * D
        dO = self.token(self.dO, H).contiguous() if tok else self.dO
        uq.uniquan_attn_window_fwd(*bw, L, D, self.Q, self.K, self.V, self.scale, self.window, self.sinks, O, lse, **how)
        Oc, lsec = O[:nq].clone(), lse[:bw[0] * L].clone()
        if tok:
            how["cs"] = self.cs = cos_sin(L)
        uq.uniquan_attn_window_bwd(*bw, L, D, self.Q, self.K, self.V, Oc, dO, lsec, self.scale, self.window, self.sinks,
                                   delta, dQ, dK, dV, **how)
        torch.cuda.synchronize()
        for t, k in ((O, nq), (lse, bw[0] * L), (delta, bw[0] * L), (dQ, nq), (dK, nq), (dV, nq)):
            assert (t[k:] == 7.0).all(), "written past the end"
        return [t[:k] for t, k in ((O, nq), (lse, bw[0] * L), (dQ, nq), (dK, nq), (dV, nq))]

    def reference(self):
        """O, lse, dQ, dK, dV (per query head, head-major) in 64 bits, and their bars before the outputs' rounding."""
        G = self.H // self.Hkv
        q, k, v, g = (t.double() for t in (self.Q, self.K.repeat(G, 1, 1), self.V.repeat(G, 1, 1), self.dO))
        see = seen_of(self.L, self.window, self.sinks)
        x = (q @ k.transpose(1, 2) * self.scale).masked_fill(~see, -math.inf)
        lse = torch.logsumexp(x, -1)
        P = (x - lse[..., None]).exp()
        O = P @ v
        ax = (q.abs() @ k.abs().transpose(1, 2) * self.scale * see).amax(-1)
        dx = (D + 16) * U * ax
        ew = (torch.expm1(2 * dx) + 2.0 ** -20)[..., None]
        n = see.sum(1).double()[:, None]
        tO = P @ v.abs() * (ew + H8 + (n + 4) * U)
        dP = g @ v.transpose(1, 2)
        tdP = (D + 4) * U * (g.abs() @ v.abs().transpose(1, 2))
        delta = (g * O).sum(-1, keepdim=True)
        tdelta = (P * (dP.abs() * (ew + (n + 4) * U) + (1 + ew) * tdP)).sum(-1, keepdim=True)
        dS = P * (dP - delta)
        tdS = dS.abs() * ew + P * (1 + ew) * (tdP + tdelta)
        tdS = tdS + H8 * (dS.abs() + tdS)
        m = self.L + 4
        dQ, tdQ = dS @ k * self.scale, (tdS + m * U * dS.abs()) @ k.abs() * self.scale
        dSt, tdSt = dS.transpose(1, 2), tdS.transpose(1, 2)
        dK, tdK = dSt @ q * self.scale, (tdSt + m * U * dSt.abs()) @ q.abs() * self.scale
        tP = (P * (ew + H8 + m * U)).transpose(1, 2)
        dV, tdV = P.transpose(1, 2) @ g, tP @ g.abs()
        tl = 1.4427 * dx + 2.0 ** -17 + 2.0 ** -22 * (lse * 1.4427).abs()
        return dict(O=(O, tO), lse=(lse / math.log(2), tl), dQ=(dQ, tdQ), dK=(dK, tdK), dV=(dV, tdV))


def turned_back(x, t, cs):
    """x [b, L, d] rotated by minus each position's angle, and the bar."""
    c, s = cs[..., 0].double(), cs[..., 1].double()
    a, b = x[..., :64], x[..., 64:]
    ta, tb = t[..., :64], t[..., 64:]
    more = 2.0 ** -22 * (a.abs() + b.abs())
    return (torch.cat([a * c + b * s, b * c - a * s], -1),
            torch.cat([ta * c.abs() + tb * s.abs() + more, tb * c.abs() + ta * s.abs() + more], -1))


def near(got, want, bar, what):
    err = (got.double() - want).abs()
    assert bool((err <= bar * 1.01 + 1e-30).all()), f"{what}: {int((err > bar).sum())} of {err.numel()} off, worst " \
        f"{float((err / (bar + 1e-30)).max()):.2f} of its bar"


def check(c, tok):
    O, lse, dQ, dK, dV = c.run(tok)
    r = c.reference()
    B, L = c.H * c.n, c.L
    near(lse.view(B, L), *r["lse"], "lse")
    outs = dict(O=O, dQ=dQ, dK=dK, dV=dV)
    for name, got in outs.items():
        want, bar = r[name]
        rounded = got.dtype == torch.bfloat16
        if tok and name in ("dQ", "dK") and rounded:
            want, bar = turned_back(want, bar, c.cs)
        if rounded:
            bar = bar + H8 * (want.abs() + bar)
        if tok and rounded:
            want, bar = c.token(want, c.H), c.token(bar, c.H)
        near(got.view(want.shape), want, bar, f"{name} at L={L}, window={c.window}, sinks={c.sinks}, tok={tok}")


@pytest.mark.parametrize("tok", [False, True])
@pytest.mark.parametrize("L", [1, 2, 31, 32, 33, 63, 100, 128, 129, 257])
def test_lengths_and_windows(L, tok):
    for window, sinks in ((1, 0), (1, 1), (2, 3), (31, 0), (32, 4), (33, 33), (100, 0), (L, 0), (L + 9, L + 5), (5, L)):
        check(Case(L, window, sinks), tok)


@pytest.mark.parametrize("tok", [False, True])
@pytest.mark.parametrize("L,window,sinks,n,H,Hkv", [
    (200, 64, 4, 2, 4, 2), (77, 10, 1, 3, 6, 2), (161, 50, 40, 2, 7, 1), (130, 200, 0, 1, 8, 8),
    (901, 600, 4, 1, 2, 1),       # walks split over two groups of wavefronts
    (1300, 512, 70, 2, 2, 2), (1024, 1, 0, 1, 2, 2), (640, 333, 129, 8, 40, 8)])
def test_heads_and_sequences(L, window, sinks, n, H, Hkv, tok):
    check(Case(L, window, sinks, n, H, Hkv), tok)


def test_large_scores():
    """Scores of a hundred and more: one key takes all the weight."""
    check(Case(150, 40, 3, size=30.0), False)


@pytest.mark.parametrize("tok", [False, True])
def test_a_window_over_everything_is_the_causal_call(tok):
    c = Case(256, 256, 0, 2, 4, 2)
    O, lse, *_ = c.run(tok)
    o2, l2 = torch.empty_like(O), torch.empty_like(lse)
    how = dict(tok_seqs=2, group=2) if tok else {}
    uq.uniquan_attn_fwd(8, 4, 256, D, c.Q, c.K, c.V, c.scale, o2, l2, **how)
    assert torch.equal(O, o2) and torch.equal(lse, l2)
    for window, sinks in ((1 << 30, 0), (2 ** 31 - 1, 2 ** 31 - 1), (3, 256), (256, 99)):
        c.window, c.sinks = window, sinks
        got = c.run(tok)
        assert torch.equal(got[0], O) and torch.equal(got[1], lse)


@pytest.mark.parametrize("name", ["Q", "K", "V"])
def test_gradients_against_differences(name):
    """The derivative of sum(O dO) along a drawn direction, from central differences of the formula in 64 bits: their
    own error is of the step's square (1e-10 here), so the bar is the gradient's along the direction."""
    c = Case(97, 20, 2, 2, 4, 2, seed=5)
    _, _, dQ, dK, dV = c.run(False)
    r = c.reference()
    got = dict(Q=dQ, K=dK, V=dV)[name].double().view(8, 97, D)
    bar = r["d" + name][1]
    G = 2
    if name != "Q":
        got, bar = got.view(G, 4, 97, D).sum(0), bar.view(G, 4, 97, D).sum(0)
    x0 = {k: getattr(c, k).double() for k in "QKV"}
    see = seen_of(97, 20, 2)
    dirn = torch.randn(x0[name].shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").double()

    def f(step):
        x = dict(x0)
        x[name] = x[name] + step * dirn
        s = (x["Q"] @ x["K"].repeat(G, 1, 1).transpose(1, 2) * c.scale).masked_fill(~see, -math.inf)
        return ((torch.softmax(s, -1) @ x["V"].repeat(G, 1, 1)) * c.dO.double()).sum()

    h = 1e-4
    want = (f(h) - f(-h)) / (2 * h)
    assert abs((got * dirn).sum() - want) <= (bar * dirn.abs()).sum() + 1e-6 * abs(want)


def test_captured_with_eager_work_between():
    c = Case(333, 50, 4, 2, 4, 2)
    B, L = 8, 333
    O, lse, delta = torch.empty(B, L, D, dtype=torch.bfloat16, device="cuda"), *(torch.empty(B, L, device="cuda") for _ in "12")
    dQ, dK, dV = (torch.empty(B, L, D, device="cuda") for _ in "123")

    def step():
        uq.uniquan_attn_window_fwd(B, 4, L, D, c.Q, c.K, c.V, c.scale, 50, 4, O, lse)
        uq.uniquan_attn_window_bwd(B, 4, L, D, c.Q, c.K, c.V, O, c.dO, lse, c.scale, 50, 4, delta, dQ, dK, dV)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        c.Q.mul_(0.9)
        c.V.add_(0.125)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (O, lse, dQ, dK, dV)]
        want = c.run(False)
        for a, b in zip(got, want):
            assert torch.equal(a.flatten(), b), f"replay {i}"


def test_strong_values_outside_the_window():
    """The largest finite keys and values where no later query looks leave those rows alone."""
    c = Case(200, 16, 0)
    O, lse, *_ = c.run(False)
    c.V[:, :32] = 3e38
    c.K[:, :32] = 1e4
    O2, lse2, *_ = c.run(False)
    late = slice(32 + 16, None)
    assert torch.equal(O.view(2, 200, D)[:, late], O2.view(2, 200, D)[:, late])
    assert torch.equal(lse.view(2, 200)[:, late], lse2.view(2, 200)[:, late])
