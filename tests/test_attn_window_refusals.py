"""Refusals of uniquan_attn_window_fwd / _bwd (no GPU)."""
import pytest

from paper_2506_03781_amd import uniquan as uq

FAKE = 1 << 20
BASE = dict(batch=4, kv_batch=2, L=33, d=128, Q=FAKE, K=FAKE, V=FAKE, scale=0.1, window=8, sinks=2, O=FAKE, lse=FAKE,
            tok=0, group=1, dO=FAKE, delta=FAKE, dQ=FAKE, dK=FAKE, dV=FAKE, cs=FAKE)


def fwd(**kw):
    a = dict(BASE, **kw)
    return uq.lib().uniquan_attn_window_fwd(a["batch"], a["kv_batch"], a["L"], a["d"], a["Q"], a["K"], a["V"], a["scale"],
                                            a["window"], a["sinks"], a["O"], a["lse"], a["tok"], a["group"], None)


def bwd(**kw):
    a = dict(BASE, **kw)
    return uq.lib().uniquan_attn_window_bwd(a["batch"], a["kv_batch"], a["L"], a["d"], a["Q"], a["K"], a["V"], a["O"],
                                            a["dO"], a["lse"], a["scale"], a["window"], a["sinks"], a["delta"], a["dQ"],
                                            a["dK"], a["dV"], a["tok"], a["group"], a["cs"], None)


BOTH = [
    (dict(window=0), uq.UQ_EINVAL, "window=0"),
    (dict(window=-3), uq.UQ_EINVAL, "window=-3"),
    (dict(sinks=-1), uq.UQ_EINVAL, "sinks=-1"),
    (dict(L=0), uq.UQ_EINVAL, "L=0"),
    (dict(L=(1 << 22) + 1), uq.UQ_EUNSUPPORTED, "L="),
    (dict(L=1 << 22, batch=256, kv_batch=256), uq.UQ_EUNSUPPORTED, "batch"),
    (dict(d=64), uq.UQ_EUNSUPPORTED, "d=64"),
    (dict(scale=0.0), uq.UQ_EINVAL, "scale"),
    (dict(scale=-1.0), uq.UQ_EINVAL, "scale"),
    (dict(scale=float("nan")), uq.UQ_EINVAL, "scale"),
    (dict(scale=float("inf")), uq.UQ_EINVAL, "scale"),
    (dict(batch=5), uq.UQ_EINVAL, "batch=5"),
    (dict(batch=65536, kv_batch=65536), uq.UQ_EUNSUPPORTED, "65535"),
    (dict(Q=None), uq.UQ_EINVAL, "Q"),
    (dict(K=FAKE + 8), uq.UQ_EINVAL, "K"),
    (dict(lse=None), uq.UQ_EINVAL, "row_lse"),
    (dict(tok=3), uq.UQ_EINVAL, "tok_seqs=3"),
    (dict(tok=2, group=0), uq.UQ_EINVAL, "group=0"),
]


@pytest.mark.parametrize("kw,status,text", BOTH)
def test_refused(kw, status, text):
    for call, name in ((fwd, "uniquan_attn_window_fwd"), (bwd, "uniquan_attn_window_bwd")):
        assert call(**kw) == status
        assert text in uq.last_error() and uq.last_error().startswith(name + ":")


@pytest.mark.parametrize("kw,text", [(dict(dO=None), "dO"), (dict(delta=None), "delta"), (dict(dQ=FAKE + 4), "dQ"),
                                     (dict(dK=None), "dK"), (dict(dV=None), "dV"), (dict(tok=2, group=2, cs=None), "cs")])
def test_backward_refused(kw, text):
    assert bwd(**kw) == uq.UQ_EINVAL
    assert text in uq.last_error()


def test_the_causal_calls_keep_their_rules():
    L = uq.lib()
    assert L.uniquan_attn_fwd(4, 2, 33, 128, FAKE, FAKE, FAKE, 0.1, FAKE, FAKE, 0, 1, None) == uq.UQ_EUNSUPPORTED
    assert "multiple of 32" in uq.last_error()
