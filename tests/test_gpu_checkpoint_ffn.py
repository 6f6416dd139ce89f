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


def test_the_largest_pre_activations():
    """Finite ones that e4m3 rounds up to 2^128: the activation goes to infinity or to zero, its slope is 1 or 0, and nothing is NaN."""
    import paper_2409_09099_amd as sste
    top = torch.finfo(torch.bfloat16).max
    H = torch.tensor([[top, -top, 3.3e38, -3.3e38] + [1.0] * 28, [float("nan"), float("inf"), float("-inf"), top] + [0.0] * 28], device="cuda").to(torch.bfloat16)
    dA = torch.full_like(H, 0.75)
    codes, scales = sste.checkpoint_pack(H)
    restored = sste.checkpoint_backward(codes, scales, act=sste.ACT_NONE)[0]
    assert torch.isinf(restored[0, :4]).all() and restored[1, 3] == float("inf") and restored[1, :3].isnan().all()
    for A, dH in (sste.checkpoint_backward(codes, scales, dA), (sste.checkpoint_backward(codes, scales)[0], sste.checkpoint_backward(codes, scales, dA, restore=False)[1])):
        assert A[0, :4].tolist() == [float("inf"), 0.0, float("inf"), 0.0] and A[1, 3] == float("inf")
        assert dH[0, :4].tolist() == [0.75, 0.0, 0.75, 0.0] and dH[1, 3] == 0.75
        assert A[1, :3].isnan().all() and dH[1, :3].isnan().all()
        assert A[0, 4:].isfinite().all() and not A[1, 4:].any() and (dH[1, 4:] == 0.375).all()
