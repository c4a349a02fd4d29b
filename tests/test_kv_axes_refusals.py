"""Refusals of uniquan_kv_append_axes (no GPU); what it shares with uniquan_kv_append is refused alike."""
import pytest
import torch

from paper_2506_03781_amd import uniquan as uq

FAKE = 1 << 20


def call(T=5, H=8, H_kv=2, d=128, q=FAKE, ld_q=0, k=FAKE, v=FAKE, dt=uq.UQ_F32, seq=None, pos=FAKE, rot=FAKE, n_axes=3,
         axis=FAKE, cs=FAKE, n_cs=10, q_out=FAKE, page_len=64):
    return uq.lib().uniquan_kv_append_axes(T, H, H_kv, d, q, ld_q, k, 0, v, 0, dt, seq, pos, rot, n_axes, axis, cs, n_cs,
                                           FAKE, 3, 4, uq.KV_BF16, 0, 9, page_len, FAKE, FAKE, None, None, q_out, None)


@pytest.mark.parametrize("kw,status,text", [
    (dict(n_axes=0), uq.UQ_EINVAL, "n_axes=0"),
    (dict(n_axes=9), uq.UQ_EINVAL, "n_axes=9"),
    (dict(rot=None), uq.UQ_EINVAL, "rot"),
    (dict(rot=FAKE + 2), uq.UQ_EINVAL, "rot"),
    (dict(axis=None), uq.UQ_EINVAL, "axis"),
    (dict(axis=FAKE + 1), uq.UQ_EINVAL, "axis"),
    (dict(cs=None), uq.UQ_EINVAL, "cs"),
    (dict(cs=FAKE + 8), uq.UQ_EINVAL, "cs"),
    (dict(n_cs=0), uq.UQ_EINVAL, "n_cs=0"),
    (dict(pos=None), uq.UQ_EINVAL, "pos"),
    (dict(d=96), uq.UQ_EUNSUPPORTED, "d=96"),
    (dict(H=7), uq.UQ_EINVAL, "H=7"),
    (dict(T=-1), uq.UQ_EINVAL, "T=-1"),
    (dict(T=1 << 30), uq.UQ_EUNSUPPORTED, "2^28"),
    (dict(q_out=None), uq.UQ_EINVAL, "q_out"),
    (dict(ld_q=1023), uq.UQ_EINVAL, "ld_q"),
    (dict(page_len=48), uq.UQ_EINVAL, "page_len"),
])
def test_refused(kw, status, text):
    assert call(**kw) == status
    assert text in uq.last_error() and uq.last_error().startswith("uniquan_kv_append_axes:")


def test_no_rows_is_ok():
    assert call(T=0, rot=None, axis=None, cs=None, k=None, v=None, pos=None) == uq.UQ_OK


def test_binding_refuses():
    x = torch.zeros(3, 128)
    with pytest.raises(TypeError, match="cs"):
        uq.uniquan_kv_append_axes(3, 1, 1, 128, x, x, x, x, x, x, None, x, x, x)
    with pytest.raises(ValueError, match="rot"):
        uq.uniquan_kv_append_axes(3, 1, 1, 128, x, x, x, x, x[:2], x, x, x, x, x)
