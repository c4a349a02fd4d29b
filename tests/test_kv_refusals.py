"""Refusals of the paged key/value cache's entry points: every bad argument is
reported on the host before anything is enqueued (no GPU)."""
import pytest
import torch

from paper_2506_03781_amd import uniquan as uq

FAKE = 1 << 20          # aligned, never dereferenced
BF, U8, U4 = uq.KV_BF16, uq.KV_U8, uq.KV_U4


@pytest.fixture(scope="module")
def L():
    return uq.lib()


def cache(a):
    st = None if a["format"] == BF else FAKE
    return (a["format"], a["group"], a["n_pages"], a["page_len"]), (a.get("k_cache", FAKE), FAKE,
                                                                    a.get("k_stat", st), a.get("v_stat", st))


BASE = dict(n_seq=3, H=8, H_kv=2, d=128, format=BF, group=0, n_pages=9, page_len=64, max_pages=4, pages=FAKE)

SHARED = [
    (dict(d=96), uq.UQ_EUNSUPPORTED, "d=96"),
    (dict(d=0), uq.UQ_EINVAL, "d=0"),
    (dict(d=256), uq.UQ_EUNSUPPORTED, "d=256"),
    (dict(format=3), uq.UQ_EINVAL, "format 3"),
    (dict(format=-1), uq.UQ_EINVAL, "format -1"),
    (dict(group=32), uq.UQ_EINVAL, "group=32"),
    (dict(format=U8, group=0), uq.UQ_EINVAL, "group=0"),
    (dict(format=U8, group=64), uq.UQ_EINVAL, "group=64"),
    (dict(format=U4, group=16), uq.UQ_EINVAL, "group=16"),
    (dict(page_len=8), uq.UQ_EINVAL, "page_len=8"),
    (dict(page_len=48), uq.UQ_EINVAL, "page_len=48"),
    (dict(page_len=2048), uq.UQ_EINVAL, "page_len=2048"),
    (dict(n_pages=0), uq.UQ_EINVAL, "n_pages=0"),
    (dict(n_pages=1 << 31), uq.UQ_EINVAL, "n_pages"),
    (dict(n_seq=0), uq.UQ_EINVAL, "n_seq=0"),
    (dict(max_pages=0), uq.UQ_EINVAL, "max_pages=0"),
    (dict(max_pages=(1 << 24) + 1), uq.UQ_EINVAL, "max_pages"),
    (dict(H_kv=0), uq.UQ_EINVAL, "H_kv=0"),
    (dict(H_kv=4097, H=4097), uq.UQ_EINVAL, "H_kv=4097"),
    (dict(pages=None), uq.UQ_EINVAL, "pages"),
    (dict(k_cache=FAKE + 8), uq.UQ_EINVAL, "k_cache"),
    (dict(format=U8, group=32, k_stat=None), uq.UQ_EINVAL, "k_stat"),
    (dict(format=U8, group=32, v_stat=FAKE + 4), uq.UQ_EINVAL, "v_stat"),
    (dict(v_stat=FAKE), uq.UQ_EINVAL, "must be NULL for bf16"),
]


def append(L, T=5, q=FAKE, ld_q=0, k=FAKE, ld_k=0, v=FAKE, ld_v=0, dt=uq.UQ_F32, seq=None, pos=FAKE, cs=None, n_cs=0,
           q_out=FAKE, **kw):
    a = dict(BASE, **kw)
    f, m = cache(a)
    return L.uniquan_kv_append(T, a["H"], a["H_kv"], a["d"], q, ld_q, k, ld_k, v, ld_v, dt, seq, pos, cs, n_cs,
                               a["pages"], a["n_seq"], a["max_pages"], *f, *m, q_out, None)


def read(L, length=5, start=None, lens=FAKE, K=FAKE, V=FAKE, dt=uq.UQ_F32, **kw):
    a = dict(BASE, **kw)
    f, m = cache(a)
    return L.uniquan_kv_read(a["n_seq"], a["H_kv"], a["d"], length, start, lens, a["pages"], a["max_pages"], *f, *m, K, V,
                             dt, None)


def attend(L, Q=FAKE, ld_q=0, lens=FAKE, O=FAKE, ld_o=0, lse=None, ws=FAKE, ws_len=1 << 40, **kw):
    a = dict(BASE, **kw)
    f, m = cache(a)
    return L.uniquan_attn_decode(a["n_seq"], a["H"], a["H_kv"], a["d"], Q, ld_q, lens, a["pages"], a["max_pages"], *f, *m,
                                 0.1, O, ld_o, lse, ws, ws_len, None)


@pytest.mark.parametrize("call", [append, read, attend])
@pytest.mark.parametrize("kw,status,text", SHARED)
def test_shared(L, call, kw, status, text):
    assert call(L, **kw) == status
    assert text in uq.last_error()


@pytest.mark.parametrize("kw,status,text", [
    (dict(H=7), uq.UQ_EINVAL, "H=7"),
    (dict(H=0), uq.UQ_EINVAL, "H=0"),
    (dict(T=-1), uq.UQ_EINVAL, "T=-1"),
    (dict(T=1 << 27), uq.UQ_EUNSUPPORTED, "2^28"),
    (dict(dt=2), uq.UQ_EINVAL, "dtype"),
    (dict(q=None), uq.UQ_EINVAL, "together"),
    (dict(q_out=None), uq.UQ_EINVAL, "together"),
    (dict(q=None, q_out=None), uq.UQ_EINVAL, "without q"),
    (dict(cs=FAKE, n_cs=0), uq.UQ_EINVAL, "n_cs"),
    (dict(ld_q=8), uq.UQ_EINVAL, "ld_q=8"),
    (dict(ld_k=260), uq.UQ_EINVAL, "ld_k=260"),
    (dict(ld_v=-8), uq.UQ_EINVAL, "ld_v"),
    (dict(k=None), uq.UQ_EINVAL, "k must not"),
    (dict(v=FAKE + 4), uq.UQ_EINVAL, "v must be 16"),
    (dict(pos=None), uq.UQ_EINVAL, "pos"),
    (dict(seq=FAKE + 2), uq.UQ_EINVAL, "seq"),
    (dict(cs=FAKE + 8, n_cs=4), uq.UQ_EINVAL, "cs"),
])
def test_append(L, kw, status, text):
    assert append(L, **kw) == status
    assert text in uq.last_error()


def test_nothing_to_do(L):
    assert append(L, T=0) == uq.UQ_OK
    assert read(L, K=None, V=None) == uq.UQ_OK


@pytest.mark.parametrize("kw,status,text", [
    (dict(length=0), uq.UQ_EINVAL, "L=0"),
    (dict(length=1 << 27), uq.UQ_EUNSUPPORTED, "2^28"),
    (dict(dt=5), uq.UQ_EINVAL, "dtype"),
    (dict(lens=None), uq.UQ_EINVAL, "lens"),
    (dict(K=FAKE + 4), uq.UQ_EINVAL, "K"),
])
def test_read(L, kw, status, text):
    assert read(L, **kw) == status
    assert text in uq.last_error()


@pytest.mark.parametrize("kw,status,text", [
    (dict(H=9), uq.UQ_EINVAL, "H=9"),
    (dict(n_seq=1 << 22), uq.UQ_EUNSUPPORTED, "2^24"),
    (dict(n_seq=1 << 13, max_pages=1 << 20), uq.UQ_EUNSUPPORTED, "2^37"),
    (dict(ld_q=1028), uq.UQ_EINVAL, "ld_q"),
    (dict(ld_o=1030), uq.UQ_EINVAL, "ld_o"),
    (dict(ld_o=512), uq.UQ_EINVAL, "ld_o"),
    (dict(Q=FAKE + 8), uq.UQ_EINVAL, "Q"),
    (dict(O=None), uq.UQ_EINVAL, "O"),
    (dict(lens=None), uq.UQ_EINVAL, "lens"),
    (dict(lse=FAKE + 2), uq.UQ_EINVAL, "row_lse"),
])
def test_attend(L, kw, status, text):
    assert attend(L, **kw) == status
    assert text in uq.last_error()


def test_workspace(L):
    """Long sequences need one; too small or misaligned is refused."""
    big = dict(max_pages=4096)
    need = uq.uniquan_attn_decode_ws(3, 8, 2, 128, 4096, 64)
    if need:
        assert attend(L, ws_len=need - 1, **big) == uq.UQ_EINVAL and "ws_len" in uq.last_error()
        assert attend(L, ws=FAKE + 4, ws_len=need, **big) == uq.UQ_EINVAL and "ws" in uq.last_error()
        assert attend(L, ws=None, ws_len=need, **big) == uq.UQ_EINVAL and "ws" in uq.last_error()
    assert uq.uniquan_attn_decode_ws(0, 8, 2, 128, 4, 64) == 0
    assert uq.uniquan_attn_decode_ws(1, 8, 2, 128, 0, 64) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    t = torch.zeros(2, 2, dtype=torch.int32)
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    with pytest.raises((ValueError, TypeError)):
        uq.uniquan_kv_append(2, 1, 1, 64, None, x, x, t[0], t, x, x)
    with pytest.raises(ValueError):
        uq.uniquan_attn_decode(2, 1, 1, 64, x, t[0], t, x, x, 0.1, x)
    with pytest.raises(ValueError):
        uq.uniquan_attn_decode(2, 1, 1, 64, x, t[0], t, x, x, 0.1, x, fmt=9)
    with pytest.raises(TypeError):
        uq.uniquan_kv_append(2, 1, 1, 64, None, None, x, t[0], t, x, x)


def test_binding_refuses_tensors_of_another_device():
    """The calls run on the current device's stream; a tensor that lies elsewhere is refused, in any argument."""
    class Far(torch.Tensor):
        is_cuda = True
        device = torch.device("cuda", 7)

    far = torch.zeros(2, 64).as_subclass(Far)
    t = torch.zeros(2, 2, dtype=torch.int32)
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    for call in (lambda: uq.uniquan_kv_append(2, 1, 1, 64, None, x, x, t[0], t, x, far),
                 lambda: uq.uniquan_kv_append(2, 1, 1, 64, None, x, x, t[0], t, x, x, cs=far),
                 lambda: uq.uniquan_kv_read(2, 1, 64, 1, t[0], t, x, x, x, far),
                 lambda: uq.uniquan_attn_decode(2, 1, 1, 64, x, t[0], t, x, x, 0.1, x, ws=far)):
        with pytest.raises(ValueError, match="cuda:7"):
            call()
