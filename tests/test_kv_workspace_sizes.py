"""uniquan_attn_decode_ws over all sizes: what the call refuses needs none, what it takes needs a size that it accepts,
however large (no GPU)."""
import pytest

from paper_2506_03781_amd import uniquan as uq

FAKE = 1 << 20  # aligned, never dereferenced: the calls here are refused before anything is enqueued


@pytest.fixture(scope="module")
def L():
    return uq.lib()


REFUSED = [
    (1 << 62, 1, 1, 128, 4096, 64), (3, 7, 2, 128, 4096, 64), (3, 8, 2, 96, 4096, 64), (3, 8, 2, 128, 4096, 48),
    (3, 8, 2, 128, 1 << 40, 64), (3, (1 << 31) - 1, 1, 128, 4096, 64), (3, (1 << 31) - 1, (1 << 31) - 1, 64, 4096, 64),
    (1 << 22, 8, 2, 128, 4, 64), (1 << 13, 8, 2, 128, 1 << 20, 64), (3, 8, 2, 128, 4, 1 << 30), (0, 8, 2, 128, 4, 64),
    (3, 8, 0, 128, 4, 64), (3, 0, 2, 128, 4, 64), (-1, 8, 2, 128, 4096, 64), (3, 8, 2, 128, -4, 64),
    (3, 8192, 4097, 128, 4096, 64),
]


@pytest.mark.parametrize("n_seq,H,H_kv,d,max_pages,page_len", REFUSED)
def test_refused_sizes(L, n_seq, H, H_kv, d, max_pages, page_len):
    assert L.uniquan_attn_decode_ws(n_seq, H, H_kv, d, max_pages, page_len) == 0
    st = L.uniquan_attn_decode(n_seq, H, H_kv, d, FAKE, 0, FAKE, FAKE, max_pages, uq.KV_BF16, 0, 9, page_len, FAKE, FAKE,
                               None, None, 0.1, FAKE, 0, None, None, 0, None)
    assert st in (uq.UQ_EINVAL, uq.UQ_EUNSUPPORTED) and "ws_len" not in uq.last_error()


@pytest.mark.parametrize("n_seq,H,H_kv,d,max_pages,page_len", [
    (1, 1, 1, 64, 1 << 26, 16), (1 << 24, 1, 1, 64, 496, 16), (3, 8, 2, 128, 4096, 64), (127, 8, 2, 128, 1 << 24, 64),
    (1, 4080, 255, 64, 1 << 20, 1024),
])
def test_least_size(L, n_seq, H, H_kv, d, max_pages, page_len):
    """The size that it states is the least that the call accepts."""
    need = L.uniquan_attn_decode_ws(n_seq, H, H_kv, d, max_pages, page_len)
    assert 0 < need < 1 << 40
    st = L.uniquan_attn_decode(n_seq, H, H_kv, d, FAKE, 0, FAKE, FAKE, max_pages, uq.KV_BF16, 0, 9, page_len, FAKE, FAKE,
                               None, None, 0.1, FAKE, 0, None, FAKE, need - 1, None)
    assert st == uq.UQ_EINVAL and "ws_len" in uq.last_error()


@pytest.mark.parametrize("n_seq,H,H_kv,d,max_pages,page_len", [
    (256, 65535, 1, 128, 4, 64), (4096, 4096, 4096, 128, 16, 64), (1, 65535, 255, 64, 1 << 20, 1024),  # one share a head
    (1 << 20, 16, 16, 64, 8, 16),  # rows of one block
])
def test_none_needed(L, n_seq, H, H_kv, d, max_pages, page_len):
    assert L.uniquan_attn_decode_ws(n_seq, H, H_kv, d, max_pages, page_len) == 0
