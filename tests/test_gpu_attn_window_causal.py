"""A window (or first positions) over everything is the causal call bit for bit, also where its walks are split over two
groups of wavefronts: few row blocks, and up to 448 of them whose longest walk is near the mean."""
import pytest
import torch

from paper_2506_03781_amd import uniquan as uq
from test_gpu_attn_window import Case, D, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tok", [False, True])
@pytest.mark.parametrize("L,n,H,Hkv", [(640, 1, 2, 1), (512, 2, 40, 8), (1024, 1, 40, 8), (1024, 5, 8, 8), (2048, 1, 18, 2),
                                       (544, 1, 3, 3), (480, 2, 2, 2)])
def test_equal_to_the_causal_call(L, n, H, Hkv, tok):
    g = torch.Generator(device="cuda").manual_seed(L + H)
    Q, K, V = (torch.randn(h * n, L, D, generator=g, device="cuda").bfloat16() for h in (H, Hkv, Hkv))
    how = dict(tok_seqs=n, group=H // Hkv) if tok else {}
    want = torch.empty_like(Q), torch.empty(H * n, L, device="cuda")
    uq.uniquan_attn_fwd(H * n, Hkv * n, L, D, Q, K, V, 0.09, *want, **how)
    for window, sinks in ((L, 0), (2 ** 31 - 1, 3), (7, L), (L - 1, L + 100)):
        got = torch.empty_like(Q), torch.empty(H * n, L, device="cuda")
        uq.uniquan_attn_window_fwd(H * n, Hkv * n, L, D, Q, K, V, 0.09, window, sinks, *got, **how)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), f"window {window}, sinks {sinks}"


@pytest.mark.parametrize("tok", [False, True])
@pytest.mark.parametrize("L,window,sinks,n,H,Hkv", [(640, 640, 0, 1, 2, 1), (700, 5, 700, 1, 3, 3), (513, 1000, 0, 8, 9, 9),
                                                    (1000, 20, 1001, 1, 40, 8)])
def test_gradients_of_a_window_over_everything(L, window, sinks, n, H, Hkv, tok):
    check(Case(L, window, sinks, n, H, Hkv), tok)


@pytest.mark.parametrize("tok", [False, True])
@pytest.mark.parametrize("L,window,sinks,n,H,Hkv", [(383, 100, 2, 1, 2, 2), (384, 100, 2, 2, 2, 1), (385, 384, 1, 1, 3, 3),
                                                    (600, 255, 0, 1, 2, 2), (600, 256, 0, 1, 4, 2), (1024, 300, 0, 2, 16, 16),
                                                    (1024, 300, 5, 3, 11, 11), (700, 1, 1, 1, 2, 1)])
def test_windows_where_the_backward_begins_to_split(L, window, sinks, n, H, Hkv, tok):
    """Longest walks of 383 to 385 rows, with and without first positions, and 256 workgroups and more."""
    check(Case(L, window, sinks, n, H, Hkv), tok)
