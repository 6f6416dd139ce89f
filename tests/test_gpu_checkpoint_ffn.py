"""The feed-forward block's backward pass from checkpoints: what it leaves to the second layer's weight gradient, and that gradient."""
import numpy as np
import pytest
import torch

from oracle import activation as OACT
from oracle import linear as OL

pytestmark = pytest.mark.gpu
BF16_STEP = torch.finfo(torch.bfloat16).eps / 2


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("T,d,h", [(192, 128, 256), (448, 320, 640)])
def test_weight_gradient_of_a_restored_activation(T, d, h):
    """A within its rounding of the float64 activation, and dW = MVUE(dY^T) A within what that rounding and float32 sums may cost, each by itself."""
    import paper_2409_09099_amd as sste
    rng = np.random.default_rng(5)
    dY = torch.from_numpy((rng.standard_normal((T, d)) * 1e-3).astype(np.float32)).to(torch.bfloat16).cuda()
    H = torch.from_numpy((rng.standard_normal((T, h)) * 1.5).astype(np.float32)).to(torch.bfloat16).cuda()
    codes, scales = sste.checkpoint_pack(H)
    A, _ = sste.checkpoint_backward(codes, scales)
    h64 = f64(sste.checkpoint_backward(codes, scales, act=sste.ACT_NONE)[0])
    a64 = OACT.gelu_tanh(h64)
    # float32 arithmetic on the hardware's exp2 and reciprocal: 1e-6 of |h|, then one rounding
    slack = 1e-6 * np.abs(h64)
    bound = slack + BF16_STEP * (np.abs(a64) + slack)
    assert (np.abs(f64(A) - a64) <= bound).all()
    theta = np.abs(OL.mvue_dense(dY.view(torch.int16).cpu().numpy().view(np.uint16), 3, 1))
    want = OL.linear_wgrad(dY.view(torch.int16).cpu().numpy().view(np.uint16), A.view(torch.int16).cpu().numpy().view(np.uint16), 3, 1)
    dW = f64(sste.linear_wgrad(dY, A, 3, 1))
    sums = (T + 16) * 2.0 ** -23 * (theta.T @ np.abs(f64(A)))             # of at most T products, in float32
    assert (np.abs(dW - want) <= sums).all()
    exact = OL.mvue_dense(dY.view(torch.int16).cpu().numpy().view(np.uint16), 3, 1).T @ a64
    assert (np.abs(dW - exact) <= sums + theta.T @ bound).all()
    assert (np.abs(dW).max(axis=1) > 0).all()
