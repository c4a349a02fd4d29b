"""Rows of another width than the cache's heads, given to the binding or to KVCache, are refused, not read as if they
lay one after the other (no GPU: the refusal comes before the library is called)."""
import pytest
import torch

from paper_2506_03781_amd import uniquan as uq
from paper_2506_03781_amd.cache import KVCache


class OnDevice(torch.Tensor):
    """A host tensor that passes for one on the device."""
    is_cuda = True
    device = torch.device("cuda", 0)


def dev(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def calls(monkeypatch):
    """The library's place taken by a list of the calls that reach it."""
    seen = []

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_ws"):
                return lambda *a: 0
            return lambda *a: seen.append(name) or 0

    monkeypatch.setattr(uq, "lib", lambda: Lib())
    monkeypatch.setattr(uq, "_stream", lambda s: 0)
    monkeypatch.setattr(uq, "_one_device", lambda *t: None)
    return seen


def cache(n_kv=2, d=64):
    c = KVCache(4, n_kv, 3, 2, d=d, page_len=16, device="cpu")
    c.k, c.v, c.table = (x.as_subclass(OnDevice) for x in (c.k, c.v, c.table))
    return c


POS = dict(dtype=torch.int32)


@pytest.mark.parametrize("k,v,q,q_out,name", [
    ((3, 136), (3, 128), None, None, "k"),
    ((3, 128), (3, 256), None, None, "v"),
    ((3, 128), (3, 128), (3, 264), (3, 256), "q"),
    ((3, 128), (3, 128), (3, 256), (3, 384), "q_out"),
    ((3, 128), (3, 128), (3, 256), (4, 200), "q_out"),
])
def test_append(calls, k, v, q, q_out, name):
    c = cache()
    with pytest.raises(ValueError, match=rf"^{name} "):
        c.append(dev(*k), dev(*v), dev(3, **POS), q=None if q is None else dev(*q),
                 q_out=None if q_out is None else dev(*q_out))
    assert not calls


@pytest.mark.parametrize("Q,O,name", [((3, 264), (3, 256), "Q"), ((3, 256), (3, 320), "O"), ((3, 256), (4, 200), "O")])
def test_attend(calls, Q, O, name):
    with pytest.raises(ValueError, match=rf"^{name} "):
        cache().attend(dev(*Q), dev(3, **POS), dev(*O))
    assert not calls


@pytest.mark.parametrize("K", [(2, 3, 6, 64), (2, 3, 5, 128), (3, 2, 5, 64)])
def test_read(calls, K):
    """K and V of another shape than [n_kv, n_seq, L, d]."""
    with pytest.raises(ValueError, match="^[KV] "):
        cache().read(dev(3, **POS), 5, dev(*K), dev(*K))
    assert not calls


@pytest.mark.parametrize("fmt,group", [("bf16", None), ("u8", 32), ("u4", 64)])
@pytest.mark.parametrize("kw", [dict(page_len=32), dict(n_kv=1), dict(n_kv=4, page_len=8), dict(d=128)])
def test_cache_of_other_sizes(calls, fmt, group, kw):
    """A cache's arrays with other heads, pages or channels than the call's."""
    c = KVCache(8, 2, 3, 2, d=64, page_len=16, fmt=fmt, group=group, device="cpu")
    m = {n: None if x is None else x.as_subclass(OnDevice)
         for n, x in dict(table=c.table, k_cache=c.k, v_cache=c.v, k_stat=c.k_stat, v_stat=c.v_stat).items()}
    n_kv, d, P = kw.get("n_kv", 2), kw.get("d", 64), kw.get("page_len", 16)
    x, lens = dev(3, n_kv * d), dev(3, **POS)
    with pytest.raises(ValueError, match="^[kv]_(cache|stat) "):
        uq.uniquan_attn_decode(3, n_kv, n_kv, d, x, lens, scale=1.0, O=dev(3, n_kv * d), page_len=P, fmt=c.fmt,
                               group=c.group, **m)
    assert not calls


@pytest.mark.parametrize("shape", [(48, 64, 2), (48, 128), (48, 16, 2)])
def test_rotary_table_of_another_head_size(calls, shape):
    with pytest.raises(ValueError, match="^cs "):
        cache().append(dev(3, 128), dev(3, 128), dev(3, **POS), cs=dev(*shape, dtype=torch.float32))
    assert not calls


def test_whole_rows_pass(calls):
    """The shapes that the calls take: rows as they are, by head, more rows than asked for, column slices, one row."""
    c = cache()
    pos = dev(3, **POS)
    wide = dev(3, 512)
    c.append(dev(3, 128), dev(3, 128), pos, cs=dev(48, 32, 2, dtype=torch.float32))
    c.append(wide[:, 8:136], wide[:, 136:264], pos, q=dev(3, 256), q_out=dev(3, 256))
    uq.uniquan_kv_append(3, 2, 2, 64, None, dev(3, 2, 64), dev(9, 128), pos, c.table, c.k, c.v, page_len=16)
    uq.uniquan_kv_append(1, 2, 2, 64, None, wide[:1, :128], dev(128), pos, c.table, c.k, c.v, page_len=16)
    uq.uniquan_kv_append(0, 2, 2, 64, None, dev(0, 128), dev(0, 128), pos, c.table, c.k, c.v, page_len=16)
    c.attend(dev(3, 256), pos, dev(3, 256))
    c.attend(wide[:, :256], pos, wide[:, 256:])
    c.read(pos, 5, dev(2, 3, 5, 64), dev(2, 3, 5, 64))
    c.read(pos, 5, dev(2 * 3 * 5 * 64), None)
    assert len(calls) == 9
