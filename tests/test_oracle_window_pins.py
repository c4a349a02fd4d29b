"""Pins of oracle.block_decoder's sliding window: which keys a query's softmax is over, entry by entry."""
import numpy as np
import pytest

import oracle.block_decoder as D


@pytest.mark.parametrize("L,window,sinks", [(1, 1, 0), (5, 1, 0), (6, 2, 1), (9, 3, 4), (7, 7, 0), (7, 20, 3), (8, 1, 8)])
def test_window_entry_by_entry(L, window, sinks):
    S = np.random.default_rng(L).standard_normal((2, L, L))
    P = D.causal_softmax(S, window, sinks)
    for b in range(2):
        for i in range(L):
            seen = [j for j in range(L) if j <= i and (i - j < window or j < sinks)]
            w = np.exp(S[b, i, seen])
            want = np.zeros(L)
            want[seen] = w / w.sum()
            assert np.allclose(P[b, i], want, rtol=1e-12, atol=0)


def test_no_window_is_causal():
    S = np.random.default_rng(0).standard_normal((6, 6))
    assert np.array_equal(D.causal_softmax(S), D.causal_softmax(S, 6, 0))
