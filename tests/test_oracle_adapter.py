"""Pins of the oracle's adapters and checkpoints: a row at a time, finite differences, and the checkpoint's guarantees."""
import numpy as np
import pytest

from oracle import adapter as OA
from oracle import checkpoint as OC
from oracle import formats as F


def test_rows_of_segments():
    ids = OA.rows_of([2, 2, 5, 7], [4, 1, -1], 3, 9)          # an empty segment, one beyond the adapters, one without; rows outside all
    assert ids.tolist() == [-1, -1, 1, 1, 1, -1, -1, -1, -1]
    assert OA.rows_of([0], [], 3, 4).tolist() == [-1] * 4
    assert OA.rows_of([0, 2, 4], [2, 3], 3, 4).tolist() == [2, 2, -1, -1]


def test_apply_row_by_row_and_gradients_by_differences():
    rng = np.random.default_rng(1)
    T, I, O, R, N = 7, 5, 6, 3, 2
    X, A, B, base, scale = rng.normal(size=(T, I)), rng.normal(size=(N, R, I)), rng.normal(size=(N, R, O)), rng.normal(size=(T, O)), np.array([0.5, 2.0])
    ids = OA.rows_of([1, 3, 4, 7], [1, 0, 1], N, T)
    Z, S, _, _ = OA.apply(X, ids, A, B, scale, base)
    for t in range(T):
        want = base[t] + (scale[ids[t]] * B[ids[t]].T @ (A[ids[t]] @ X[t]) if ids[t] >= 0 else 0)
        assert np.allclose(Z[t], want, rtol=1e-13)
    assert not S[ids < 0].any()
    dZ = rng.normal(size=(T, O))
    loss = lambda X, A, B: float((OA.apply(X, ids, A, B, scale, base)[0] * dZ).sum())      # noqa: E731
    dX, dS, _, _ = OA.apply(dZ, ids, B, A, scale, None)
    dA, dB = OA.outer(dS, X, ids, N)[0], OA.outer(S, dZ, ids, N)[0]
    h = 1e-5
    for value, grad, at in ((X, dX, (3, 2)), (X, dX, (0, 1)), (A, dA, (1, 2, 4)), (A, dA, (0, 0, 0)), (B, dB, (1, 1, 5)), (B, dB, (0, 2, 3))):
        kept = value[at]
        value[at] = kept + h
        up = loss(X, A, B)
        value[at] = kept - h
        down = loss(X, A, B)
        value[at] = kept
        assert abs((up - down) / (2 * h) - grad[at]) < 1e-8
    assert dX[0].max() == 0 == np.abs(dX[0]).max()


def test_checkpoint_blocks():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(40, 112)) * np.exp2(rng.integers(-140, 120, size=(40, 4)).astype(float)).repeat(32, axis=1)[:, :112]
    x = F.bf16_to_f32(F.f32_to_bf16_rne(x.astype(np.float32))).astype(np.float64)
    codes, scales = OC.pack(x)
    back = OC.decode(codes, scales)
    step = np.exp2(scales.astype(float) - 127).repeat(32, axis=1)[:, :112]
    assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step)).all()
    for b in range(4):                                        # the least exponent: one less would not hold the block
        top, e = np.abs(x[:, b * 32:b * 32 + 32]).max(axis=1), scales[:, b].astype(int) - 127
        assert (top <= 448 * np.exp2(e.astype(float))).all() and ((e == -117) | (top > 448 * np.exp2(e - 1.0))).all()


@pytest.mark.parametrize("top,e", [(448.0, 0), (450.0, 1), (447.0, 0), (0.0, -117), (1.0, -8), (1.75, -8), (1.7578125, -7), (2.0 ** -126, -117)])
def test_checkpoint_exponent(top, e):
    codes, scales = OC.pack(np.array([[top] + [0.0] * 15]))
    assert scales.tolist() == [[e + 127]]
    assert abs(OC.decode(codes, scales)[0, 0] - top) <= 2.0 ** -4 * top


def test_checkpoint_non_finite():
    codes, scales = OC.pack(np.array([[np.inf, -np.inf, np.nan, 3.0] + [0.0] * 12]))
    assert codes[0, :3].tolist() == [0x7F] * 3 and OC.decode(codes, scales)[0, 3] == 3.0
