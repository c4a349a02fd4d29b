"""DecoderBlock(window, sinks) at odd sequence lengths (the tokens of all sequences a multiple of 32), also where the
projections write the heads in the products' store; bars as in test_gpu_window_block."""
import numpy as np
import pytest
import torch

import oracle.block_decoder as D
import test_gpu_decoder_block as B
from paper_2506_03781_amd import uniquan as uq
from test_gpu_window_block import F32, bf16, block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,H,n_kv,L,n_seq,window,sinks", [(256, 2, 1, 33, 32, 7, 1), (256, 2, 2, 3, 64, 2, 0),
                                                           (256, 2, 2, 97, 32, 97, 0), (1024, 8, 4, 129, 128, 40, 3)])
def test_step_against_the_oracle(C, H, n_kv, L, n_seq, window, sinks):
    T = L * n_seq
    X, mats, g1, g2 = B.make_block(L, qk_scale=3.0, shapes=B.shapes_for(C, 384, n_kv * 128), T_=T)
    blk, qs = block(mats, g1, g2, T, n_seq, H, n_kv, window, sinks)
    if C == 1024:  # the products of 256 tiles and more
        assert -(-T // 256) * -(-C // 256) >= 256 and blk._stacked_kv({n: qs[n].W_hat for n in qs}) is not None
    W = {n: np.asarray(m[0], F32) for n, m in mats.items()}
    how = dict(n_kv=n_kv, window=window, sinks=sinks, store=bf16)
    ref = D.decoder_forward(X, W, g1, g2, n_seq, H, **how)["Y"]
    blk.prepare(X)
    Y = B.share_target(blk, ref)
    blk.set_input(X)
    blk.forward_backward(uq.MAP_FULL)
    torch.cuda.synchronize()
    what = {n: B.host(qs[n].W_hat) for n in mats}
    st = D.decoder_step(X, Y, what, g1, g2, n_seq, H, **how)
    assert abs(float(blk.loss.item()) - st["loss"]) <= 1e-2 * st["loss"]
    for n in mats:
        x, want = B.host(qs[n].G), st["grads"][n]
        off = np.linalg.norm(x - want) / np.linalg.norm(want)
        assert off <= 1e-2, f"{n}: {off}"


def test_tokens_that_are_no_multiple_of_32_are_refused():
    X, mats, g1, g2 = B.make_block(1, shapes=B.shapes_for(256, 384, 256), T_=33)
    with pytest.raises(AssertionError, match="multiples of 32"):
        block(mats, g1, g2, 33, 1, 2, 2, 7, 0)
