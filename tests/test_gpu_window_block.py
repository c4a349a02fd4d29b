"""A decoder block with a sliding window (DecoderBlock(window, sinks)) against oracle.block_decoder with the same
window: the loss and dL/dWhat of all seven matrices within 1e-2 normwise, the bar of the block without one."""
import numpy as np
import pytest
import torch

import oracle.block_decoder as D
import oracle.uniquan as O
import test_gpu_decoder_block as B
from paper_2506_03781_amd import uniquan as uq
from paper_2506_03781_amd.block import DecoderBlock, QuantMatrix

pytestmark = pytest.mark.gpu
F32 = np.float32


def bf16(x):
    return O.bf16_rne(np.asarray(x, F32)).astype(np.float64)


def block(mats, g1, g2, T, n_seq, H, n_kv, window, sinks):
    qs = {n: QuantMatrix(W, s, B.K, B.G, p["delta"], p["z_u"], p["s_r"], p["z_b"], p["alpha"])
          for n, (W, s, p) in mats.items()}
    return DecoderBlock(qs, g1, g2, T, n_seq, H, n_kv=n_kv, window=window, sinks=sinks), qs


@pytest.mark.parametrize("C,H,n_kv,L,n_seq,window,sinks", [(256, 2, 2, 64, 2, 20, 2), (256, 2, 2, 48, 4, 9, 0),
                                                           (512, 4, 2, 80, 2, 33, 40)])
def test_step_against_the_oracle(C, H, n_kv, L, n_seq, window, sinks):
    T = L * n_seq
    X, mats, g1, g2 = B.make_block(7, qk_scale=3.0, shapes=B.shapes_for(C, 384, n_kv * 128), T_=T)
    blk, qs = block(mats, g1, g2, T, n_seq, H, n_kv, window, sinks)
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



def test_recorded_steps_repeat():
    """step_fused recorded once and replayed: the same parameters as as many eager steps."""
    X, mats, g1, g2 = B.make_block(3)
    got = []
    for recorded in (False, True):
        blk, qs = block(mats, g1, g2, B.T, B.N_SEQ, B.H, 2, 20, 2)
        blk.prepare(X)
        blk.set_input(X)
        blk.quantize(uq.MAP_FULL)
        step = lambda: blk.step_fused(uq.MAP_LOCAL, 1e-5, 1e-6)  # noqa: E731
        if recorded:
            call = uq.record(step)
            call()
            call()
        else:
            for _ in range(3):
                step()
        torch.cuda.synchronize()
        got.append({n: (q.s.clone(), q.alpha.clone(), q.W_hat.clone()) for n, q in qs.items()})
    for n in got[0]:
        assert all(torch.equal(a, b) for a, b in zip(got[0][n], got[1][n])), n
