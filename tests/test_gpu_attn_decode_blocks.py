"""uniquan_attn_decode on long rows whose answer shows every block of positions, within bars that a lost or misplaced
block breaks (attend_bars)."""
import numpy as np
import pytest
import torch

from attend_bars import LONG, attend, bars, broken, long_rows, queries
from kv_cases import FORMS, attend_bounds, filled, rounded
from paper_2506_03781_amd import uniquan as uq

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    uq.lib()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def check(c, q, lens, scale):
    O, lse = attend(c, q, lens, scale)
    el, norm = broken(O, c, q, lens, scale, bars(c, q, lens, scale))
    assert not el.any() and not norm.any(), (np.argwhere(el)[:5], np.argwhere(norm)[:5])
    want, tol = attend_bounds(c, q, lens, scale)[1::2]
    empty = ~np.isfinite(want)
    assert np.all(lse[empty] == -np.inf) and np.all(O[empty] == 0)
    assert np.all(np.abs(lse[~empty] - want[~empty]) <= tol[~empty])


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("d,n_kv,grp,P", [(128, 1, 4, 64), (64, 1, 12, 16), (128, 1, 12, 32), (64, 2, 8, 256)])
@pytest.mark.parametrize("shown", [True, False])
def test_every_block(fmt, group, d, n_kv, grp, P, shown):
    """Rows split into many chunks, some of them ending inside a share, beside short and empty ones."""
    rs = np.random.default_rng(90 + grp + d)
    c = long_rows(rs, LONG, n_kv, d, P, fmt, group, shown)
    check(c, queries(rs, len(LONG), n_kv * grp, d), LONG, d ** -0.5)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("shown", [True, False])
def test_few_shares(fmt, group, shown):
    """Many key/value heads, so that each has few shares: chunks of many blocks over several sequences' ends."""
    rs = np.random.default_rng(95)
    lens = [700, 1, 1300, 0, 128, 129, 2500, 40]
    c = long_rows(rs, lens, 120, 64, 64, fmt, group, shown)
    check(c, queries(rs, len(lens), 240, 64), lens, 0.125)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("grp", [3, 16])
def test_holes(fmt, group, grp):
    """Every third page is none: the blocks that are left count as they do without the others."""
    rs = np.random.default_rng(96)
    lens = [3000, 640, 129]
    c = long_rows(rs, lens, 1, 128, 32, fmt, group, True)
    c.table[:, 1::3] = -1
    check(c, queries(rs, 3, grp, 128), lens, 0.09)


@pytest.mark.parametrize("fmt,group", FORMS)
@pytest.mark.parametrize("grp", [4, 12])
def test_keys_with_a_large_channel(fmt, group, grp):
    """One key channel ten times the others', whose offset makes the scores of codes large sums."""
    rs = np.random.default_rng(97)
    lens = [3000, 777, 31]
    c = filled(rs, lens, 1, 128, 64, fmt, group)
    check(c, rounded(rs, 3, grp, 128), lens, 0.088)
