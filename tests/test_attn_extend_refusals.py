"""Refusals of uniquan_attn_extend and its workspace query (no GPU)."""
import pytest

from paper_2506_03781_amd import uniquan as uq

FAKE = 1 << 20
BASE = dict(T=5, n_seq=3, H=8, H_kv=2, d=128, Q=FAKE, ld_q=0, row_start=FAKE, lens=FAKE, mask=None, words=0, pos=None,
            window=0, sinks=0, pages=FAKE, max_pages=4, fmt=uq.KV_BF16, group=0, n_pages=9, page_len=64, k=FAKE, v=FAKE,
            ks=None, vs=None, scale=0.1, O=FAKE, ld_o=0, lse=None, ws=FAKE, ws_len=1 << 40)


def call(**kw):
    a = dict(BASE, **kw)
    return uq.lib().uniquan_attn_extend(
        a["T"], a["n_seq"], a["H"], a["H_kv"], a["d"], a["Q"], a["ld_q"], a["row_start"], a["lens"], a["mask"], a["words"],
        a["pos"], a["window"], a["sinks"], a["pages"], a["max_pages"], a["fmt"], a["group"], a["n_pages"], a["page_len"],
        a["k"], a["v"], a["ks"], a["vs"], a["scale"], a["O"], a["ld_o"], a["lse"], a["ws"], a["ws_len"], None)


@pytest.mark.parametrize("kw,status,text", [
    (dict(T=-1), uq.UQ_EINVAL, "T=-1"),
    (dict(T=1 << 31), uq.UQ_EINVAL, "T="),
    (dict(T=(1 << 23) + 1), uq.UQ_EUNSUPPORTED, "2^26"),
    (dict(n_seq=0), uq.UQ_EINVAL, "n_seq=0"),
    (dict(n_seq=1 << 22), uq.UQ_EUNSUPPORTED, "2^24"),
    (dict(H=7), uq.UQ_EINVAL, "H=7"),
    (dict(d=96), uq.UQ_EUNSUPPORTED, "d=96"),
    (dict(page_len=8), uq.UQ_EINVAL, "page_len"),
    (dict(max_pages=0), uq.UQ_EINVAL, "max_pages"),
    (dict(fmt=3), uq.UQ_EINVAL, "format"),
    (dict(fmt=uq.KV_U8, group=64, ks=FAKE, vs=FAKE), uq.UQ_EINVAL, "group=64"),
    (dict(fmt=uq.KV_U8, group=32), uq.UQ_EINVAL, "k_stat"),
    (dict(ld_q=1023), uq.UQ_EINVAL, "ld_q"),
    (dict(ld_q=1028), uq.UQ_EINVAL, "ld_q"),
    (dict(ld_o=1026), uq.UQ_EINVAL, "ld_o"),
    (dict(window=-1), uq.UQ_EINVAL, "window=-1"),
    (dict(sinks=-1), uq.UQ_EINVAL, "sinks=-1"),
    (dict(mask=FAKE, words=0), uq.UQ_EINVAL, "words=0"),
    (dict(mask=FAKE, words=65), uq.UQ_EINVAL, "words=65"),
    (dict(mask=FAKE + 4, words=1), uq.UQ_EINVAL, "mask"),
    (dict(mask=FAKE, words=1, window=9), uq.UQ_EINVAL, "positions"),
    (dict(pos=FAKE + 2), uq.UQ_EINVAL, "pos"),
    (dict(Q=None), uq.UQ_EINVAL, "Q"),
    (dict(Q=FAKE + 8), uq.UQ_EINVAL, "Q"),
    (dict(row_start=None), uq.UQ_EINVAL, "row_start"),
    (dict(lens=None), uq.UQ_EINVAL, "lens"),
    (dict(O=FAKE + 4), uq.UQ_EINVAL, "O"),
    (dict(lse=FAKE + 2), uq.UQ_EINVAL, "row_lse"),
    (dict(max_pages=1000, ws_len=10), uq.UQ_EINVAL, "ws_len=10"),
    (dict(max_pages=1000, ws=None), uq.UQ_EINVAL, "ws"),
    (dict(max_pages=1000, ws=FAKE + 4), uq.UQ_EINVAL, "ws"),
])
def test_refused(kw, status, text):
    assert call(**kw) == status
    assert text in uq.last_error() and uq.last_error().startswith("uniquan_attn_extend:")


def test_no_rows_is_ok():
    assert call(T=0, Q=None, row_start=None, lens=None, O=None, ws=None, ws_len=0) == uq.UQ_OK


def test_workspace():
    ws = uq.uniquan_attn_extend_ws
    assert ws(1, 1, 32, 8, 128, 1000, 64) > 0
    assert ws(1, 1, 32, 8, 128, 1, 64) == 0                 # no sequence is long enough to be cut
    assert ws(100000, 1, 32, 8, 128, 1000, 64) == 0         # tiles enough
    for bad in ((0, 1, 32, 8, 128, 9, 64), (-1, 1, 32, 8, 128, 9, 64), (5, 0, 32, 8, 128, 9, 64), (5, 1, 33, 8, 128, 9, 64),
                (5, 1, 32, 8, 100, 9, 64), (5, 1, 32, 8, 128, 9, 60), (1 << 27, 1, 32, 8, 128, 9, 64)):
        assert ws(*bad) == 0, bad
