"""uniquan_attn_extend_ws over numbers of key/value heads (no GPU): a tile is cut into two shares or more, or not at all."""
import pytest

from paper_2506_03781_amd import uniquan as uq

FEWEST = 16  # columns of a share


@pytest.mark.parametrize("T,n_seq", [(1, 1), (3, 2), (40, 5), (300, 4), (2000, 9), (70000, 300)])
@pytest.mark.parametrize("grp", [1, 4, 15])
@pytest.mark.parametrize("d", [64, 128])
def test_room_for_two_shares_or_none(T, n_seq, grp, d):
    for n_kv in (1, 2, 3, 8, 85, 127, 128, 129, 170, 171, 255, 256, 257, 300, 320, 511, 512, 513, 1000, 4096):
        need = uq.uniquan_attn_extend_ws(T, n_seq, n_kv * grp, n_kv, d, 100, 64)
        if n_kv > 256:
            assert need == 0, f"{n_kv} heads: a GPU of 512 places holds no two workgroups of each"
        else:
            assert need == 0 or need >= 2 * FEWEST * n_kv * (d + 4), n_kv
