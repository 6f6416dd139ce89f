"""Adapter products whose every intermediate is a small integer: float32 holds all of them, so results are equal to the formula's bit for bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sste():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_09099_amd as lib
    lib.library()
    return lib


def launches(sste, call):
    """(result, launches of adapter kernels)."""
    sste.timing_begin(64)
    try:
        result = call()
    finally:
        times = sste.timing_end()
    return result, times["adapter"][1]


FORMATS = {"bf16": (torch.bfloat16, "BF16"), "e4m3": (torch.float8_e4m3fn, "F8E4M3"), "e5m2": (torch.float8_e5m2, "F8E5M2")}


# rows, width in, width out, rank, launches
SIZES = [(1, 64, 8, 8, 1), (70, 144, 520, 16, 1), (100, 272, 264, 32, 1), (129, 528, 136, 64, 1), (65, 592, 264, 128, 1),
         (3000, 5120, 1032, 16, 2), (3000, 5120, 1032, 32, 2), (700, 2064, 136, 64, 2), (8300, 208, 1032, 64, 1), (9000, 272, 136, 64, 2), (700, 2064, 136, 128, 2), (5003, 2064, 136, 120, 2)]


@pytest.mark.parametrize("T,K,C,R,count", SIZES)
@pytest.mark.parametrize("fwd,kind", [(True, "bf16"), (True, "e4m3"), (False, "bf16"), (False, "e4m3"), (False, "e5m2")])
def test_every_bit_of_the_low_rank_product_counts(sste, T, K, C, R, count, fwd, kind):
    """S has 24 bits in one rank and their upper 18, negative, in another; their sum, the lower 6 bits, is the output.

    Digits of three bits are exact in every format, and powers of two in bf16, so S is an integer below 2^24 in whatever order its terms are added.  What
    the second product adds up, parts of the two ranks, are multiples of 1 below 2^24 and cancel to less: also exact in any order, and the sum of 6 bits is
    one of bf16's numbers.  A representation of S by fewer than 24 bits shows as another result."""
    rng = np.random.default_rng(T + R)
    dtype, name = FORMATS[kind]
    digits = rng.integers(0, 8, (T, 8))
    digits[:, 7] |= 4                                                     # 24 bits
    at = rng.permutation(K)[:8]
    X = np.zeros((T, K))
    X[:, at] = digits
    down, up = np.zeros((2, R, K)), np.zeros((2, R, C))
    full, upper = rng.permutation(R)[:2]
    down[1, full, at] = 8.0 ** np.arange(8)
    down[1, upper, at[2:]] = -(8.0 ** np.arange(2, 8))
    up[1, [full, upper]] = 1.0
    down[0], up[0] = 3.0, 5.0                                             # an adapter that nobody has
    v = (digits * 8 ** np.arange(8)).sum(1)
    low = digits[:, 0] + 8 * digits[:, 1]
    gpu = lambda a, t=torch.bfloat16: torch.from_numpy(a.astype(np.float32)).cuda().to(t)      # noqa: E731
    rows = torch.tensor([0, T // 2, T], dtype=torch.int32, device="cuda"), torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    x, a, b = gpu(X, dtype), gpu(down), gpu(up)
    call = (lambda: sste.adapter_fwd(x, *rows, a, b, dtype=getattr(sste, name))) if fwd else (lambda: sste.adapter_dgrad(x, *rows, b, a, dtype=getattr(sste, name)))
    (out, S), number = launches(sste, call)
    assert number == count
    want = np.zeros((T, R))
    want[:, full], want[:, upper] = v, low - v
    assert np.array_equal(S.cpu().numpy(), want)
    assert np.array_equal(out.float().cpu().numpy(), np.repeat(low[:, None], C, 1))


def test_products_with_the_largest_floats(sste):
    """S is the largest float32 in one row: it enters the second product as it is, not as the infinity that bf16 rounds it to."""
    T, K, C, R = 20, 64, 136, 16
    X, A, B = torch.zeros((T, K), device="cuda"), torch.zeros((1, R, K), device="cuda"), torch.zeros((1, R, C), device="cuda")
    X[3, :8] = 7 * 2.0 ** 52                                              # eight digits of three bits: 2^24 - 1, times 2^104
    A[0, 5, :8] = 2.0 ** 52 * 8.0 ** torch.arange(8, device="cuda")
    B[0, 5] = 2.0 ** -104
    X, A, B = (t.to(torch.bfloat16) for t in (X, A, B))
    rows = torch.tensor([0, T], dtype=torch.int32, device="cuda"), torch.tensor([0], dtype=torch.int32, device="cuda")
    Z, S = sste.adapter_fwd(X, *rows, A, B)
    assert S[3, 5] == torch.finfo(torch.float32).max and S.count_nonzero() == 1
    assert (Z[3] == 2.0 ** 24).all() and not Z[:3].any() and not Z[4:].any()
    dX, dS = sste.adapter_dgrad(X, *rows, B, A)
    assert torch.equal(dX, Z) and torch.equal(dS, S)


@pytest.mark.parametrize("T", [400, 2400])                               # in one launch and in two
def test_gradients_of_every_exponent(sste, T):
    """S = (1 + 2^-23) 2^e: both its bits arrive, up to the largest floats and down to 2^-110 (its last bit is then the smallest bf16)."""
    R, I, O = 8, 64, 72
    exponents = np.arange(-110, 128)
    N = len(exponents)
    value, other = (torch.from_numpy(np.ldexp(m, n)).cuda() for m, n in ((1 + 2.0 ** -23, exponents), (1.0, -exponents.clip(-100, 100))))      # exactly: on the host
    S = torch.zeros((T, R), device="cuda")
    S[:N, 3] = value.float()
    S[N - 1, 4] = torch.finfo(torch.float32).max
    M = torch.zeros((T, O), device="cuda")
    M[:N] = other.float()[:, None]
    M = M.to(torch.bfloat16)
    starts = torch.arange(N + 1, dtype=torch.int32, device="cuda")
    ids = torch.arange(N, dtype=torch.int32, device="cuda")
    dA, dB = sste.adapter_wgrad(M, M[:, :I].contiguous(), S, S, starts, ids, N)
    want = torch.zeros((N, R), device="cuda", dtype=torch.float64)
    want[:, 3] = value * other
    want[N - 1, 4] = torch.finfo(torch.float32).max * other[N - 1]
    for G in (dA, dB):
        wrong = (G.double() != want[:, :, None]).any(2).any(1)
        assert not wrong.any(), exponents[wrong.cpu().numpy()]
