"""8-bit activation checkpoints on the GPU against the oracle: the pack bit for bit, the backward pass within its roundings."""
import numpy as np
import pytest
import torch

from oracle import activation as OACT
from oracle import checkpoint as OC

pytestmark = pytest.mark.gpu
BF16_STEP = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module")
def sste():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_09099_amd as lib
    lib.library()
    return lib


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def values(T, C, seed=0, spread=8):
    """bf16 values whose blocks have magnitudes of their own."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, C)) * np.exp2(rng.integers(-spread, spread + 1, (T, (C + 31) // 32)).astype(float)).repeat(32, axis=1)[:, :C]
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()


SIZES = [(1, 16), (1, 1280), (3, 48), (17, 1296), (333, 80), (64, 5120), (1, 16400), (5, 8192 + 16), (2049, 32), (1100, 64)]


@pytest.mark.parametrize("T,C", SIZES)
def test_pack_bits(sste, T, C):
    X = values(T, C)
    codes, scales = sste.checkpoint_pack(X)
    want_codes, want_scales = OC.pack(f64(X))
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)


def test_pack_every_magnitude(sste):
    """Every finite bf16 as the largest of a block, with smaller ones of the same and of lower exponents beside it; and each sign."""
    bits = np.arange(0x7F80, dtype=np.uint16)
    top = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).double().numpy()
    x = np.zeros((len(bits), 32))
    x[:, 7] = -top
    x[:, 20] = top * 0.7
    x[:, 21] = top * 2.0 ** -9
    x[:, 31] = -top * 2.0 ** -15
    X = torch.from_numpy(x).float().to(torch.bfloat16).cuda()
    codes, scales = sste.checkpoint_pack(X)
    want_codes, want_scales = OC.pack(f64(X))
    assert np.array_equal(scales.cpu().numpy(), want_scales) and np.array_equal(codes.cpu().numpy(), want_codes)
    H, _ = sste.checkpoint_backward(codes, scales, act=sste.ACT_NONE)
    back = OC.decode(want_codes, want_scales)
    back = np.where(np.abs(back) >= 2.0 ** 128, np.copysign(np.inf, back), back)
    assert np.array_equal(f64(H), back)


def test_pack_non_finite(sste):
    X = values(8, 96)
    X[0, 0], X[1, 33], X[2, 64], X[2, 65] = float("inf"), float("nan"), float("-inf"), 5.0
    X[3, :32] = float("nan")
    codes, scales = sste.checkpoint_pack(X)
    want_codes, want_scales = OC.pack(f64(X))
    got = codes.cpu().numpy()
    got = np.where((got & 0x7F) == 0x7F, 0x7F, got)                      # a NaN code of either sign
    assert np.array_equal(scales.cpu().numpy(), want_scales) and np.array_equal(got, want_codes)
    A, dH = sste.checkpoint_backward(codes, scales, dA=torch.ones_like(X))
    assert torch.equal(torch.isnan(A), ~torch.isfinite(X)) and torch.equal(torch.isnan(dH), ~torch.isfinite(X))


def check_backward(sste, T, C, act, restore, grad, in_place=False, pad=0, seed=0):
    rng = np.random.default_rng(seed)

    def room(t):
        """The matrix with `pad` columns of room behind its rows."""
        r = torch.full((t.shape[0], t.shape[1] + pad), 77, dtype=t.dtype, device="cuda")
        r[:, :t.shape[1]] = t
        return r, r[:, :t.shape[1]]

    codes0, scales0 = sste.checkpoint_pack(values(T, C, seed, 3))
    (rc, codes), (rs, scales) = room(codes0), room(scales0)
    rd, dA = room(torch.from_numpy((rng.standard_normal((T, C)) * 1e-3).astype(np.float32)).to(torch.bfloat16).cuda())
    d64 = f64(dA)
    ra, A = room(torch.zeros((T, C), dtype=torch.bfloat16, device="cuda"))
    got = sste.checkpoint_backward(codes, scales, dA=dA if grad else None, act=act, A=A if restore else None, dH=dA if in_place else None, restore=restore)
    h = OC.decode(codes0.cpu().numpy(), scales0.cpu().numpy())
    gelu = act == sste.ACT_GELU_TANH
    if restore:
        want = OACT.gelu_tanh(h) if gelu else h
        # float32 arithmetic on the hardware's exp2 and reciprocal: 1e-6 of |h| (GELU is h times a sigmoid), then one rounding
        slack = 1e-6 * np.abs(h) if gelu else 0.0
        assert (np.abs(f64(got[0]) - want) <= slack + BF16_STEP * (np.abs(want) + slack)).all()
    else:
        assert got[0] is None
    if grad:
        slope = OACT.gelu_tanh_grad(h) if gelu else np.ones_like(h)
        slack = 2e-6 * np.abs(d64) if gelu else 0.0                        # about 1e-6 absolute in the derivative
        assert (np.abs(f64(got[1]) - d64 * slope) <= slack + BF16_STEP * (np.abs(d64 * slope) + slack)).all()
    else:
        assert got[1] is None
    for r in (rc, rs, ra) + ((rd,) if in_place else ()):
        if pad:
            assert (r[:, -pad:] == 77).all()


@pytest.mark.parametrize("T,C", SIZES)
@pytest.mark.parametrize("act,restore,grad", [(1, True, True), (0, True, False)])
def test_backward(sste, T, C, act, restore, grad):
    check_backward(sste, T, C, act, restore, grad)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("restore,grad,in_place,pad", [(True, True, False, 16), (False, True, False, 0), (False, True, True, 16), (True, False, False, 16), (True, True, True, 0)])
def test_backward_outputs_and_strides(sste, act, restore, grad, in_place, pad):
    check_backward(sste, 65, 144, act, restore, grad, in_place, pad)


def test_pack_strides_and_far_rows(sste):
    """Rows of a wider buffer; row offsets beyond 2^32 bytes."""
    X = values(600, 144)
    want = sste.checkpoint_pack(X)
    wide = torch.empty((600, 1 << 22), dtype=torch.bfloat16, device="cuda")          # 5 GB, used in its first columns only
    wide[:, :144] = X
    codes = torch.empty((600, 1 << 23), dtype=torch.uint8, device="cuda")[:, :144]
    scales = torch.empty((600, 11), dtype=torch.uint8, device="cuda")[:, 3:8]
    got = sste.checkpoint_pack(wide[:, :144], codes, scales)
    assert got[0] is codes and torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    A, _ = sste.checkpoint_backward(codes, scales, act=sste.ACT_NONE, A=wide[:, 256:400])
    assert torch.equal(A, sste.checkpoint_backward(*want, act=sste.ACT_NONE)[0])


def test_empty(sste):
    for shape in ((0, 64), (5, 0)):
        X = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        codes, scales = sste.checkpoint_pack(X)
        A, dH = sste.checkpoint_backward(codes, scales, dA=X)
        assert codes.shape == A.shape == dH.shape == shape


def test_gelu_ends(sste):
    """Large pre-activations and zeros: 0 or the value itself, slopes 0, 1/2 and 1, no NaN."""
    X = torch.tensor([[-3e38, -1e4, -448.0, -10.0, -0.0, 0.0, 10.0, 448.0, 1e4, 3e38] + [0.0] * 6], dtype=torch.bfloat16, device="cuda").t().contiguous().expand(16, 16).contiguous()
    codes, scales = sste.checkpoint_pack(X)
    H, dH = sste.checkpoint_backward(codes, scales, dA=torch.ones_like(X))
    h = sste.checkpoint_backward(codes, scales, act=sste.ACT_NONE)[0]
    assert torch.equal(H[:3], torch.zeros_like(H[:3])) and torch.equal(H[7:10], h[7:10])
    assert (dH[:3] == 0).all() and (dH[4:6] == 0.5).all() and (dH[7:10] == 1).all()


def test_ffn_backward_from_checkpoints(sste):
    """The feed-forward block's backward pass with its pre-activations in 8 bits: what fc2's weight gradient and fc1's backward read.  Bitwise the same as the
    restored pre-activations through the block's own fused input gradient wherever both round once, and within a rounding elsewhere."""
    rng = np.random.default_rng(5)
    T, d, h = 192, 128, 256
    W = torch.from_numpy((rng.standard_normal((d, h)) * 0.02).astype(np.float32)).to(torch.bfloat16).cuda()
    dY = torch.from_numpy((rng.standard_normal((T, d)) * 1e-3).astype(np.float32)).to(torch.bfloat16).cuda()
    H = values(T, h, 6, 1)
    vals, meta = sste.project_pack(W, 1.4830322)
    codes, scales = sste.checkpoint_pack(H)
    g = sste.linear_dgrad(dY, vals, meta, h)
    A, dH = sste.checkpoint_backward(codes, scales, dA=g)
    back = sste.checkpoint_backward(codes, scales, act=sste.ACT_NONE)[0]
    fused = sste.linear_dgrad_act(dY, vals, meta, h, back)
    # both round g to bf16 and the product to bf16: a slope 2e-6 apart moves a result by at most that and one more rounding
    assert (np.abs(f64(dH) - f64(fused)) <= 2 * BF16_STEP * np.abs(f64(fused)) + 4e-6 * np.abs(f64(g))).all()
    dW = sste.linear_wgrad(dY, A, 3, 1)
    assert torch.equal(dW, sste.linear_wgrad(dY, torch.from_numpy(OACT.gelu_tanh(f64(back)).astype(np.float32)).to(torch.bfloat16).cuda(), 3, 1)) or \
        (np.abs(f64(A) - OACT.gelu_tanh(f64(back))) <= 1e-6 * np.abs(f64(back)) + BF16_STEP * (np.abs(f64(A)) + 1e-6)).all()


def test_graph(sste):
    X, dA = values(100, 144), values(100, 144, 1)
    codes, scales = sste.checkpoint_pack(X)
    A, dH = torch.empty_like(X), torch.empty_like(X)

    def step():
        sste.checkpoint_pack(X, codes, scales)
        sste.checkpoint_backward(codes, scales, dA=dA, A=A, dH=dH)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        X.copy_(values(100, 144, 10 + k))
        step()
        want = [t.clone() for t in (codes, scales, A, dH)]
        for t in (codes, scales, A, dH):
            t.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((codes, scales, A, dH), want)), k
