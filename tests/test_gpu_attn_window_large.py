"""uniquan_attn_window_fwd / _bwd on operands of more than 2^32 elements: the last sequence as it comes out alone."""
import pytest
import torch

from paper_2506_03781_amd import uniquan as uq
from test_gpu_attn_window import D, cos_sin

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tok", [False, True])
def test_offsets_past_32_bits(tok):
    L, n, window, sinks = (1 << 21) + 5, 17, 40, 2
    assert n * L * D > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(0)

    def call(q, k, v, do, m):
        how = dict(tok_seqs=m, group=1) if tok else {}
        O, lse, delta = torch.empty_like(q), torch.empty(m, L, device="cuda"), torch.empty(m, L, device="cuda")
        grads = [torch.empty_like(q, dtype=torch.bfloat16 if tok else torch.float32) for _ in range(3)]
        uq.uniquan_attn_window_fwd(m, m, L, D, q, k, v, 0.09, window, sinks, O, lse, **how)
        if tok:
            how["cs"] = cs
        uq.uniquan_attn_window_bwd(m, m, L, D, q, k, v, O, do, lse, 0.09, window, sinks, delta, *grads, **how)
        torch.cuda.synchronize()
        return [O, lse, *grads]

    cs = cos_sin(L) if tok else None
    ops = [torch.empty(n, L, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(4)]
    full = call(*ops, n)
    for s in (0, n - 1):
        alone = call(*(t[s:s + 1].contiguous() for t in ops), 1)
        for name, a, b in zip(("O", "lse", "dQ", "dK", "dV"), full, alone):
            assert torch.equal(a[s:s + 1], b), f"{name} of sequence {s}"
