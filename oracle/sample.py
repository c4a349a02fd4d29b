"""Plain reference of uniquan_sample: one token per row of logits (numpy, one
row at a time, integer weights as Python integers)."""
import math

import numpy as np


def shift(V):
    return min(51, 62 - max(0, math.ceil(math.log2(V))))


def weights(x, t, sh):
    """Integer weights of a row of fp32 values: round(e^((x - max) / t) 2^sh)."""
    top = x.max()
    w = []
    for v in x.astype(np.longdouble):
        if v == top:
            w.append(1 << sh)
        elif v == -np.inf or np.isinf(top):
            w.append(0)
        else:
            w.append(int(np.rint(np.exp((v - np.longdouble(top)) / np.longdouble(t)) * np.longdouble(2.0) ** sh)))
    return w


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob, the kept indices in order of value) of one row x [V] (fp32 values)."""
    x = np.where(np.isnan(x), -np.inf, x).astype(np.float32)
    V = len(x)
    if x.max() == -np.inf:
        return -1, 0.0, []
    order = sorted(range(V), key=lambda i: (-x[i], i))
    if not temperature > 0:
        return order[0], 1.0, order[:1]
    sh = shift(V)
    w = weights(x, np.float32(temperature), sh)
    if 0 < top_k < V:
        order = order[:top_k]
    if top_p < 1:
        total, before, kept = sum(w[i] for i in order), 0, []
        p = int(np.float64(np.float32(top_p)) * 2.0 ** 64) if top_p > 0 else 0
        for i in order:
            if kept and not before << 64 < p * total:
                break
            kept.append(i)
            before += w[i]
        order = kept
    if min_p > 0:
        least = min(np.float64(np.float32(min_p)), 1.0) * 2.0 ** sh
        order = [i for i in order if w[i] >= least]
    total = sum(w[i] for i in order)
    at = total - 1 if u >= 1 else (int(np.float64(np.float32(u)) * 2.0 ** 64) * total >> 64) if u > 0 else 0
    run = 0
    for i in sorted(order):
        run += w[i]
        if run > at:
            return i, w[i] / total, order
    raise AssertionError("no token")
