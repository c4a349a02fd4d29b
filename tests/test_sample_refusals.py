"""Refusals of uniquan_sample (no GPU), and pins of its plain reference."""
import numpy as np
import pytest
import torch

from oracle.sample import sample_row, shift, weights
from paper_2506_03781_amd import uniquan as uq

FAKE = 1 << 20


def call(T=3, V=100, logits=FAKE, ld=0, dt=uq.UQ_F32, u=FAKE, temperature=None, top_k=None, top_p=None, min_p=None,
         token=FAKE, prob=None, ws=FAKE, ws_len=1 << 40):
    return uq.lib().uniquan_sample(T, V, logits, ld, dt, u, temperature, top_k, top_p, min_p, token, prob, ws, ws_len, None)


@pytest.mark.parametrize("kw,status,text", [
    (dict(T=-1), uq.UQ_EINVAL, "T=-1"),
    (dict(T=1 << 31), uq.UQ_EINVAL, "T="),
    (dict(V=0), uq.UQ_EINVAL, "V=0"),
    (dict(V=(1 << 22) + 1), uq.UQ_EUNSUPPORTED, "V="),
    (dict(ld=99), uq.UQ_EINVAL, "ld=99"),
    (dict(dt=2), uq.UQ_EINVAL, "dtype"),
    (dict(logits=None), uq.UQ_EINVAL, "logits"),
    (dict(logits=FAKE + 8), uq.UQ_EINVAL, "logits"),
    (dict(u=None), uq.UQ_EINVAL, "u "),
    (dict(token=None), uq.UQ_EINVAL, "token"),
    (dict(token=FAKE + 2), uq.UQ_EINVAL, "token"),
    (dict(prob=FAKE + 1), uq.UQ_EINVAL, "prob"),
    (dict(temperature=FAKE + 1), uq.UQ_EINVAL, "temperature"),
    (dict(top_k=FAKE + 2), uq.UQ_EINVAL, "top_k"),
    (dict(top_p=FAKE + 2), uq.UQ_EINVAL, "top_p"),
    (dict(min_p=FAKE + 2), uq.UQ_EINVAL, "min_p"),
])
def test_refused(kw, status, text):
    assert call(**kw) == status
    assert text in uq.last_error() and "uniquan_sample" in uq.last_error()


def test_no_rows_is_ok():
    assert call(T=0, logits=None, u=None, token=None) == uq.UQ_OK


def test_workspace_of_refused_sizes_is_0():
    assert uq.uniquan_sample_ws(-1, 5) == uq.uniquan_sample_ws(3, 0) == uq.uniquan_sample_ws(3, 1 << 23) == 0


def test_binding_refuses():
    x = torch.zeros(3, 5)
    with pytest.raises(ValueError, match="device tensor"):
        uq.uniquan_sample(3, 5, x, x, x)
    with pytest.raises(TypeError, match="logits"):
        uq.uniquan_sample(3, 5, None, x, x)


def test_reference_weights_and_shift():
    assert [shift(v) for v in (1, 2, 1024, 1025, 131072, 1 << 22)] == [51, 51, 51, 51, 45, 40]
    w = weights(np.array([0.0, -np.log(2.0), -np.inf], np.float32), 1.0, 51)
    assert w[0] == 1 << 51 and abs(w[1] - 2 ** 50) < 2 ** 29 and w[2] == 0


def test_reference_filters_in_turn():
    x = np.log(np.array([0.1, 0.4, 0.3, 0.2], np.float32))
    assert sample_row(x, 0.0, top_k=2)[2] == [1, 2]
    assert sample_row(x, 0.0, top_p=0.65)[2] == [1, 2]
    assert sample_row(x, 0.0, top_k=2, top_p=0.5)[2] == [1]          # of the two: 0.57 and 0.43
    assert sample_row(x, 0.0, min_p=0.6)[2] == [1, 2]
    assert sample_row(x, 0.0, top_p=0.0)[2] == [1]
    assert sample_row(x, 0.99)[0] == 3 and sample_row(x, 0.05)[0] == 0 and sample_row(x, 0.2)[0] == 1
    assert sample_row(np.array([1, 1, 1, 1], np.float32), 0.5, top_k=3)[2] == [0, 1, 2]
    assert sample_row(x, 0.7, temperature=0.0)[:2] == (1, 1.0)
    assert sample_row(np.full(4, np.nan, np.float32), 0.5)[0] == -1
