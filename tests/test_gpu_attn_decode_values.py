"""uniquan_attn_decode over the whole range of what a cache can hold: infinite
values, against oracle/kv_cache.py in 64 bits with bars from
kv_cases.attend_bounds."""
import copy

import numpy as np
import pytest
import torch

import oracle.kv_cache as KV
from kv_cases import attend_bounds, dev, filled, on_device, rounded
from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu
F32 = np.float32
INF = 0x7F80  # bf16 bits; with the sign 0xFF80


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    uq.lib()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def attend(c, q, lens, scale):
    """O [n, H, d] and the log-sum-exp [n, H] in 64 bits, from the device."""
    n, H, d = q.shape
    m = on_device(c)
    O = torch.full((n, H * d), float("nan"), device="cuda", dtype=torch.bfloat16)
    lse = torch.full((n, H), float("nan"), device="cuda")
    ws = torch.full((max(1, uq.uniquan_attn_decode_ws(n, H, c.n_kv, d, m["table"].shape[1], c.P)),), float("nan"),
                    device="cuda")
    uq.uniquan_attn_decode(n, H, c.n_kv, d, dev(q.reshape(n, H * d)).bfloat16(), dev(np.asarray(lens, np.int32)),
                           scale=scale, O=O, row_lse=lse, ws=ws, **m)
    torch.cuda.synchronize()
    return O.float().cpu().numpy().astype(np.float64).reshape(n, H, d), lse.cpu().numpy().astype(np.float64)


def within(got, want, tol, what=""):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, NaN {np.isnan(got).sum()}"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("grp", [1, 8, 12])
@pytest.mark.parametrize("scale", [0.0, 0.1])
def test_infinite_values(d, grp, scale):
    """A channel with an infinite value at a position in use is that infinity, whatever the position's weight (the
    largest, any other, all alike); with both signs it is NaN.  Other channels and other heads are not touched, nor
    are rows with the same values behind their length."""
    rs = np.random.default_rng(40 + grp)
    lens = [1, 40, 300, 2500, 20]
    c = filled(rs, lens, 2, d, 16, "bf16", 0, outlier=False)
    q = rounded(rs, len(lens), 2 * grp, d)
    clean = copy.deepcopy(c)
    want = {}
    for s, ln in enumerate(lens):
        top = int(np.argmax(clean.dense(s, ln)[0][1] @ q[s, grp].astype(np.float64)))  # the first head's top position
        places = [(0, top, INF), (3, ln - 1, INF | 0x8000), (d // 2 + 5, ln // 2, INF), (d - 1, 0, INF | 0x8000)]
        if s == 4:
            places = [(ch, ln, b) for ch, _, b in places]  # the first position that is not the sequence's
        elif ln > 1:
            places += [(9, 0, INF), (9, ln - 1, INF | 0x8000)]
        for ch, p, b in places:
            c.v[c.page(s, p), 1, p % 16, ch] = b
            clean.v[c.page(s, p), 1, p % 16, ch] = 0
            if s != 4:
                want[s, ch] = np.nan if ch == 9 else -np.inf if b & 0x8000 else np.inf
    O, lse = attend(c, q, lens, scale)
    ref, ref_l, tol, tol_l = attend_bounds(clean, q, lens, scale)
    for (s, ch), x in want.items():
        assert np.array_equal(O[s, grp:, ch], np.full(grp, x), equal_nan=True), (s, ch, O[s, grp:, ch])
        O[s, grp:, ch] = ref[s, grp:, ch] = 0
    within(O, ref, tol)
    within(lse, ref_l, tol_l)
