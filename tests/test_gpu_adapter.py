"""Low-rank adapters on the GPU against the oracle, element by element, within what float32 accumulation and the roundings may cost."""
import numpy as np
import pytest
import torch

from oracle import adapter as OA
from oracle import checkpoint as OC

pytestmark = pytest.mark.gpu
BF16_STEP = torch.finfo(torch.bfloat16).eps / 2          # half a step, relative


@pytest.fixture(scope="module")
def sste():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_09099_amd as lib
    lib.library()
    return lib


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def normal(rng, shape, std):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).cuda()


def stored(sste, t, kind, pad=0):
    """(tensor with `pad` columns of room behind each row, its float64 values, dtype constant, scale)."""
    T, C = t.shape
    if kind == "bf16":
        room = torch.full((T, C + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        room[:, :C] = t.to(torch.bfloat16)
        return room[:, :C], f64(room[:, :C]), sste.BF16, 1.0
    dtype = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[kind]
    scale = float(t.abs().max()) / torch.finfo(dtype).max if t.numel() else 1.0
    codes = (t / scale).to(dtype)
    room = torch.full((T, C + pad), 0x7F, dtype=torch.uint8, device="cuda")      # NaN behind the rows
    room[:, :C] = codes.view(torch.uint8)
    return room[:, :C], f64(codes) * float(np.float32(scale)), {"e4m3": sste.F8E4M3, "e5m2": sste.F8E5M2}[kind], scale


def segments(starts, ids):
    return torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(ids, dtype=torch.int32, device="cuda")


def within(name, got, want, bound):
    """|got - want| <= bound for every element."""
    err = np.abs(f64(got) - want)
    bad = ~(err <= bound)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4], err[bad][:4], np.broadcast_to(bound, err.shape)[bad][:4])


def check_apply(sste, fwd, T, K, C, R, N, starts, ids, kind, base=True, scale=True, in_place=False, pad=0, seed=0, workspace=None):
    rng = np.random.default_rng(seed)
    X, x64, dt, xs = stored(sste, normal(rng, (T, K), 1.0), kind, pad)
    down, up = (torch.full((N, R, w + pad), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :, :w].copy_(normal(rng, (N, R, w), 0.05)) for w in (K, C))
    s = normal(rng, (N,), 1.0) if scale else None
    b = stored(sste, normal(rng, (T, C), 1.0), "bf16", pad)[0] if base else None
    b64 = None if b is None else f64(b)
    row_start, seg = segments(starts, ids)
    rows = OA.rows_of(starts, ids, N, T)
    out64, S64, eS, eO = OA.apply(x64, rows, f64(down), f64(up), None if s is None else f64(s), b64)
    if fwd:
        out, S = sste.adapter_fwd(X, row_start, seg, down, up, scale=s, base=b, dtype=dt, x_scale=xs, Z=b if in_place else None, workspace=workspace)
    else:
        out, S = sste.adapter_dgrad(X, row_start, seg, up, down, scale=s, base=b, dtype=dt, dy_scale=xs, dX=b if in_place else None, workspace=workspace)
    torch.cuda.synchronize()
    within("S", S, S64, eS)
    within("out", out, out64, eO + BF16_STEP * (np.abs(out64) + eO))
    if (rows < 0).any():
        none = torch.from_numpy(rows < 0).cuda()
        assert not S[none].any()
        want = torch.from_numpy(b64[rows < 0]).cuda() if base else torch.zeros_like(out[none]).double()
        assert torch.equal(out[none].double(), want)


# one token; a decode batch; rows around the tiles of 16 and 64; widths around the steps of 64 and 128; every rank's padding
SHAPES = [
    (1, 64, 8, 8, 1, [0, 1], [0]),
    (1, 1280, 3840, 16, 5, [0, 1], [3]),
    (15, 136, 520, 16, 3, [0, 15], [2]),
    (17, 72, 128, 24, 3, [0, 1, 17], [1, 0]),
    (33, 200, 1032, 32, 4, [0, 16, 16, 33], [3, 1, 0]),
    (70, 264, 144, 40, 4, [3, 3, 40, 66], [3, -1, 2]),            # rows outside all segments, an empty one, one without
    (129, 1032, 264, 64, 2, [0, 64, 128, 129], [1, 0, 1]),
    (200, 328, 648, 96, 3, [0, 100, 200], [7, 1]),                # an adapter that is not there
    (257, 520, 392, 128, 2, [0, 250], [1]),
    (48, 8, 8, 8, 1, [0, 48], [0]),
]


@pytest.mark.parametrize("fwd", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s[:5]))
def test_bf16(sste, shape, fwd):
    check_apply(sste, fwd, *shape, "bf16")


@pytest.mark.parametrize("T,K,C,R", [(1, 16, 8, 8), (19, 144, 520, 16), (130, 1296, 136, 48), (65, 592, 264, 128), (700, 2064, 136, 64), (3000, 5120, 1032, 16), (3000, 5120, 1032, 32)])
@pytest.mark.parametrize("fwd,kind", [(True, "e4m3"), (False, "e4m3"), (False, "e5m2")])
def test_8_bit(sste, T, K, C, R, fwd, kind):
    check_apply(sste, fwd, T, K, C, R, 3, [0, T // 2, T], [2, 0], kind)


@pytest.mark.parametrize("R", [8, 16, 24, 32, 64, 128])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,K,C", [(8300, 208, 264), (4300, 2064, 264), (3100, 5120, 1032)])
def test_long_batches(sste, R, kind, T, K, C):
    """Many rows, in tiles of 16, 32 and (long contractions) of 64, ragged segments among them."""
    check_apply(sste, True, T, K, C, R, 3, [5, 70, 134, 199, T - 100], [2, -1, 0, 1], kind, seed=R)


@pytest.mark.parametrize("T,K,C,R", [(3000, 5120, 1032, 8), (3000, 5120, 1032, 32), (700, 2056, 136, 64), (700, 5120, 136, 64), (700, 2056, 136, 128), (700, 5120, 136, 128)])
@pytest.mark.parametrize("fwd", [True, False])
def test_split_contraction(sste, T, K, C, R, fwd):
    """The first product shared out among workgroups, into a workspace; without one, or with one that is too small, not shared out."""
    need = sste.adapter_workspace_bytes(T, 3, R, K, C)
    assert need > 0 and need % (T * R * 4) == 0
    for workspace in (None, torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(need - 1, dtype=torch.uint8, device="cuda"),
                      torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")):
        check_apply(sste, fwd, T, K, C, R, 3, [0, 133, 600, 690], [2, -1, 0], "bf16", workspace=workspace)


@pytest.mark.parametrize("base,scale,in_place,pad", [(False, True, False, 0), (True, False, False, 16), (True, True, True, 16), (False, False, False, 0), (True, True, True, 0)])
@pytest.mark.parametrize("T,K,C,R", [(37, 144, 136, 16), (8200, 144, 136, 16), (3000, 5120, 1032, 16), (700, 2056, 136, 64), (5000, 2056, 136, 128)])
def test_base_scale_strides(sste, base, scale, in_place, pad, T, K, C, R):
    check_apply(sste, True, T, K, C, R, 3, [0, 9, 20, T - 4], [1, -1, 2], "bf16", base, scale, in_place, pad)


@pytest.mark.parametrize("S", [63, 64, 65, 200, 4100, 5000])
def test_many_segments(sste, S):
    """The search of a tile takes one, two and three rounds; empty segments among them."""
    rng = np.random.default_rng(S)
    T = 1500
    starts = np.sort(rng.integers(0, T + 1, S + 1)).tolist()
    check_apply(sste, True, T, 64, 64, 8, 9, starts, rng.integers(-1, 9, S).tolist(), "bf16")


@pytest.mark.parametrize("T,K,R", [(74, 5120, 16), (75, 5120, 16), (6003, 1280, 64), (6004, 1280, 64), (621, 1024, 128), (622, 1024, 128), (2787, 1024, 128), (2788, 1024, 128), (1848, 2056, 64),
                                   (1849, 2056, 64), (4324, 2056, 64), (4325, 2056, 64), (5003, 2056, 128), (8192, 2056, 128)])
def test_around_the_plans_ends(sste, T, K, R):
    """Sizes on both sides of every choice between the ways of sharing the products out."""
    check_apply(sste, True, T, K, 136, R, 2, [0, T // 3, T], [1, 0], "bf16")


def test_a_million_empty_segments(sste):
    S = 1 << 20
    for T, K, R in ((1, 64, 8), (70, 5120, 64)):                                        # in one launch and in two
        check_apply(sste, True, T, K, 7168, R, 2, [0] * S + [1], [0] * (S - 1) + [1], "bf16")


@pytest.mark.parametrize("T,I,O,R", [(9, 64, 72, 8), (8200, 64, 72, 8), (700, 2056, 136, 64)])          # in one launch, and in two with a shared contraction
def test_empty(sste, T, I, O, R):
    """No rows, no segments, no adapters, no columns."""
    rng = np.random.default_rng(0)
    X, A, B = normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (2, R, I), 1).to(torch.bfloat16), normal(rng, (2, R, O), 1).to(torch.bfloat16)
    base = normal(rng, (T, O), 1).to(torch.bfloat16)
    rs, sa = segments([0], [])
    Z, S = sste.adapter_fwd(X, rs, sa, A, B, base=base)
    assert torch.equal(Z, base) and not S.any()
    rs, sa = segments([0, T], [0])
    Z, S = sste.adapter_fwd(X, rs, sa, A[:0], B[:0], base=base)
    assert torch.equal(Z, base) and not S.any()
    Z, S = sste.adapter_fwd(X[:0], rs, sa, A, B)
    assert Z.shape == (0, O) and S.shape == (0, R)
    Z, S = sste.adapter_fwd(X[:, :0], rs, sa, A[:, :, :0], B, base=base)
    assert torch.equal(Z, base) and not S.any()
    Z, S = sste.adapter_fwd(X, rs, sa, A, B[:, :, :0])
    want = OA.apply(f64(X), OA.rows_of([0, T], [0], 2, T), f64(A), f64(B[:, :, :0]), None, None)
    within("S", S, want[1], want[2])


@pytest.mark.parametrize("T,I,O,R", [(5, 64, 72, 8), (8200, 64, 72, 8), (700, 2056, 136, 64)])
def test_no_segments_need_no_arrays(sste, T, I, O, R):
    """segments = 0 through the C ABI, with NULL for both arrays."""
    rng = np.random.default_rng(4)
    X, base = normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (T, O), 1).to(torch.bfloat16)
    A, B = normal(rng, (2, R, I), 1).to(torch.bfloat16), normal(rng, (2, R, O), 1).to(torch.bfloat16)
    Z, S = torch.full_like(base, 7), torch.full((T, R), 7.0, device="cuda")
    dA, dB = torch.full((2, R, I), 7.0, device="cuda"), torch.full((2, R, O), 7.0, device="cuda")
    ws = torch.empty(sste.adapter_wgrad_workspace_bytes(T, 0, R, I, O), dtype=torch.uint8, device="cuda")
    lib, p, stream = sste.library(), lambda t: t.data_ptr(), torch.cuda.current_stream().cuda_stream      # noqa: E731
    assert lib.sste_adapter_fwd(p(X), T, I, I, 0, 1.0, None, 0, None, p(A), I, p(B), O, None, 2, R, O, p(base), O, p(Z), O, p(S), R, None, 0, stream) == 0
    assert lib.sste_adapter_wgrad(p(base), T, O, O, 0, 1.0, p(X), I, I, 0, 1.0, None, 0, p(S), R, p(S), R, None, 0, None, 2, R, p(dA), I, p(dB), O, 0, p(ws), ws.numel(), stream) == 0
    assert torch.equal(Z, base) and not S.any() and not dA.any() and not dB.any()


@pytest.mark.parametrize("T,I,O,R", [(40, 64, 72, 8), (8200, 64, 72, 8), (700, 2056, 136, 64)])
def test_malformed_segments_stay_inside(sste, T, I, O, R):
    """Bounds beyond the rows are clamped, and bounds that decrease leave the memory around the outputs alone."""
    rng = np.random.default_rng(1)
    X, A, B = normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (2, R, I), 1).to(torch.bfloat16), normal(rng, (2, R, O), 1).to(torch.bfloat16)
    room_z = torch.full((T + 32, O + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    room_s = torch.full((T + 32, R + 4), 7.0, dtype=torch.float32, device="cuda")
    Z, S = room_z[16:-16, :O], room_s[16:-16, :R]
    for starts, ids in (([-5, 20, T + 100], [0, 1]), ([30, 10, T], [0, 1]), ([2 ** 31 - 1, -2 ** 31, 5, 2 ** 31 - 1], [0, 1, 0])):
        rs, sa = segments(starts, ids)
        sste.adapter_fwd(X, rs, sa, A, B, Z=Z, S=S)
        torch.cuda.synchronize()
        for room, w in ((room_z, O), (room_s, R)):
            assert (room[:16] == 7).all() and (room[-16:] == 7).all() and (room[:, w:] == 7).all()
        need = sste.adapter_wgrad_workspace_bytes(T, len(ids), R, I, O)
        ws, room_g = torch.full((need + 256,), 0x11, dtype=torch.uint8, device="cuda"), torch.full((4, R, I), 7.0, device="cuda")
        sste.adapter_wgrad(Z, X, S, S, rs, sa, 2, dA=room_g[1:3], workspace=ws[:need])
        assert (ws[need:] == 0x11).all() and (room_g[0] == 7).all() and (room_g[3] == 7).all()
    rs, sa = segments([-5, 20, T + 100], [0, 1])
    got, want = sste.adapter_fwd(X, rs, sa, A, B), sste.adapter_fwd(X, *segments([0, 20, T], [0, 1]), A, B)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("T,I,O,R", [(40, 128, 136, 16), (8200, 128, 136, 16), (700, 2056, 136, 64)])
def test_rows_keep_to_themselves(sste, T, I, O, R):
    """A row's infinities and NaN reach no other row, an adapter's no row of another adapter; a row's result does not depend on the other rows."""
    rng = np.random.default_rng(2)
    X, A, B = normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (3, R, I), 1).to(torch.bfloat16), normal(rng, (3, R, O), 1).to(torch.bfloat16)
    seg = segments([0, 10, 21, T], [0, 1, 0])
    Z0, S0 = sste.adapter_fwd(X, *seg, A, B)
    X2, A2 = X.clone(), A.clone()
    X2[5, 7], X2[30, 0], X2[T - 1, 127] = float("nan"), float("inf"), float("-inf")
    A2[1], A2[2] = float("nan"), float("nan")
    Z1, S1 = sste.adapter_fwd(X2, *seg, A2, B)
    hit = torch.zeros(T, dtype=torch.bool, device="cuda")
    hit[[5, 30, T - 1]] = True
    hit[10:21] = True
    assert torch.equal(Z0[~hit], Z1[~hit]) and torch.equal(S0[~hit], S1[~hit])
    assert not torch.isfinite(Z1[hit].float()).any(dim=1).all() and not torch.isfinite(S1[hit]).any()


@pytest.mark.parametrize("T", [600, 2100])
def test_far_rows(sste, T):
    """Row offsets beyond 2^32 bytes: a view of a large buffer with long rows."""
    ld = 1 << 22
    rng = np.random.default_rng(3)
    room = torch.empty((T, ld), dtype=torch.bfloat16, device="cuda")              # 5 and 18 GB, read and written in its first columns only
    x, base = normal(rng, (T, 72), 1).to(torch.bfloat16), normal(rng, (T, 80), 1).to(torch.bfloat16)
    A, B = normal(rng, (2, 8, 72), 1).to(torch.bfloat16), normal(rng, (2, 8, 80), 1).to(torch.bfloat16)
    room[:, :72], room[:, 128:208] = x, base
    seg = segments([0, T // 2, T], [1, 0])
    Z, S = sste.adapter_fwd(room[:, :72], *seg, A, B, base=room[:, 128:208], Z=room[:, 256:336])
    want = sste.adapter_fwd(x, *seg, A, B, base=base)
    assert torch.equal(Z, want[0]) and torch.equal(S, want[1])
    g, w = torch.zeros((2, 8, 72), device="cuda"), torch.zeros((2, 8, 80), device="cuda")
    dA, dB = sste.adapter_wgrad(room[:, 256:336], room[:, :72], S, S, *seg, 2)
    dA2, dB2 = sste.adapter_wgrad(want[0], x, S, S, *seg, 2, dA=g, dB=w)
    assert torch.equal(dA, dA2) and torch.equal(dB, dB2)


# ---- weight gradients -----------------------------------------------------------------------------------------------
def check_wgrad(sste, T, I, O, R, N, starts, ids, kind="bf16", x_kind="bf16", accumulate=False, pad=0, seed=0):
    rng = np.random.default_rng(seed)
    dZ, dz64, dt, dzs = stored(sste, normal(rng, (T, O), 1e-3), kind, pad)
    blocks = None
    if x_kind == "checkpoint":
        X, blocks = sste.checkpoint_pack(normal(rng, (T, I), 1.0).to(torch.bfloat16))
        x64, xdt, xs = OC.decode(X.cpu().numpy(), blocks.cpu().numpy()), sste.F8BLOCK, 1.0
    else:
        X, x64, xdt, xs = stored(sste, normal(rng, (T, I), 1.0), x_kind, pad)
    rows = OA.rows_of(starts, ids, N, T)
    S, dS = normal(rng, (T, R), 1.0), normal(rng, (T, R), 1e-3)
    if pad:
        S, dS = (torch.cat([v, torch.full((T, 4), float("nan"), device="cuda")], 1)[:, :R] for v in (S, dS))
    S[torch.from_numpy(rows < 0).cuda()] = float("nan")                  # not read where there is no adapter
    dA = dB = None
    kept = [0.0, 0.0]
    if accumulate:
        dA, dB = normal(rng, (N, R, I), 1.0), normal(rng, (N, R, O), 1.0)
        kept = [f64(dA), f64(dB)]
    row_start, seg = segments(starts, ids)
    dA, dB = sste.adapter_wgrad(dZ, X, S, dS, row_start, seg, N, dtype=dt, dy_scale=dzs, x_dtype=xdt, x_scale=xs, x_blocks=blocks, dA=dA, dB=dB, accumulate=accumulate)
    torch.cuda.synchronize()
    A64, eA = OA.outer(f64(dS), x64, rows, N)
    B64, eB = OA.outer(np.where(rows[:, None] < 0, 0, f64(S)), dz64, rows, N)
    for name, got, want, bound, old in (("dA", dA, A64, eA, kept[0]), ("dB", dB, B64, eB, kept[1])):
        within(name, got, want + old, bound + OA.ACCUMULATE * (np.abs(want) + np.abs(old)) * 2)
    if not accumulate:
        for n in set(range(N)) - set(rows.tolist()):
            assert not dA[n].any() and not dB[n].any()


@pytest.mark.parametrize("T,I,O,R,N,starts,ids", [
    (1, 64, 8, 8, 2, [0, 1], [1]),
    (31, 136, 520, 16, 3, [0, 31], [2]),
    (33, 8, 264, 24, 2, [0, 1, 33], [1, 0]),
    (129, 72, 128, 32, 3, [0, 64, 64, 129], [2, 1, 2]),            # an adapter twice, one empty
    (300, 392, 136, 64, 2, [10, 200, 280], [1, -1]),
    (1000, 128, 264, 128, 4, [0, 500, 900, 1000], [3, 9, 0]),
    (8200, 200, 144, 16, 3, [0, 1, 4000, 8100], [2, 0, 2]),
    (8200, 1032, 72, 48, 1, [0, 8200], [0]),
    (95, 264, 512, 40, 2, [0, 63, 95], [1, 0]),                    # around the 64 rows of a step, and their halves
    (97, 256, 520, 72, 2, [0, 32, 97], [1, 0]),
    (2000, 136, 72, 96, 9, sorted(i * 7919 % 2001 for i in range(201)), [i % 10 for i in range(200)]),
    (2047, 72, 264, 16, 2, [0, 100, 2040], [1, 0]),                # on both sides of the few rows that are one launch: rows
    (2048, 264, 128, 40, 3, [0, 127, 128, 2048], [2, 1, 2]),
    (2049, 136, 72, 40, 3, [0, 127, 128, 2049], [2, 1, 2]),
    (511, 136, 72, 8, 3, [0, 255, 256, 511], [2, 1, 2]),
    (513, 136, 72, 8, 3, [0, 1, 512, 513], [2, 1, 2]),
    (256, 64, 136, 24, 5, list(range(257)), [i * 3 % 6 for i in range(256)]),                # segments
    (256, 64, 136, 24, 5, [0] + list(range(257)), [i * 3 % 6 for i in range(257)]),
    (256, 200, 16, 128, 1, sorted(i * 617 % 257 for i in range(257)), [0] * 256),
    (250, 16, 200, 48, 3, sorted(i * 617 % 257 for i in range(257)), [i % 3 for i in range(256)]),
    (70, 24, 40, 56, 2, [3, 3, 36, 36, 68], [0, 1, 0, 0]),
    (2500, 392, 136, 64, 2, [10, 1200, 1280], [1, -1]),            # the same small sizes in chunks
    (2100, 8, 264, 24, 2, [0, 1, 33], [1, 0]),
    (2300, 136, 520, 16, 3, [0, 31], [2]),
])
def test_wgrad(sste, T, I, O, R, N, starts, ids):
    check_wgrad(sste, T, I, O, R, N, starts, ids)


@pytest.mark.parametrize("kind,x_kind", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e5m2", "checkpoint"), ("bf16", "checkpoint")])
@pytest.mark.parametrize("R", [8, 32, 64, 128])
@pytest.mark.parametrize("T", [333, 2333])
def test_wgrad_8_bit(sste, kind, x_kind, R, T):
    check_wgrad(sste, T, 208, 400, R, 3, [0, 100, 200, T - 13], [2, 0, 2], kind, x_kind)


@pytest.mark.parametrize("accumulate,pad", [(True, 0), (True, 16), (False, 16)])
@pytest.mark.parametrize("T", [500, 2500])
def test_wgrad_accumulates_and_strides(sste, accumulate, pad, T):
    check_wgrad(sste, T, 144, 272, 16, 3, [0, 100, T], [2, 0], accumulate=accumulate, pad=pad)


@pytest.mark.parametrize("T", [100, 2300])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_wgrad_keeps_to_its_rows(sste, T, kind):
    """NaN in the rows of one adapter, of none and of no segment reach no other adapter's gradients."""
    rng = np.random.default_rng(6)
    X, _, dt, xs = stored(sste, normal(rng, (T, 144), 1), kind)
    dZ, S, dS = normal(rng, (T, 80), 1).to(torch.bfloat16), normal(rng, (T, 40), 1), normal(rng, (T, 40), 1)
    seg = segments([5, 17, 40, 66, T - 20], [1, 0, -1, 2])
    want = sste.adapter_wgrad(dZ, X, S, dS, *seg, 3, x_dtype=dt, x_scale=xs)
    for part in (slice(0, 17), slice(40, 66), slice(T - 20, T)):
        for t in (dZ, S, dS):
            t[part] = float("nan")
        X[part] = float("nan") if kind == "bf16" else 0x7F
    dA, dB = sste.adapter_wgrad(dZ, X, S, dS, *seg, 3, x_dtype=dt, x_scale=xs)
    for n in (0, 2):
        assert torch.equal(dA[n], want[0][n]) and torch.equal(dB[n], want[1][n])
    assert dA[1].isnan().all() and dB[1].isnan().all()


def test_wgrad_empty(sste):
    rs, sa = segments([0, 0], [0])
    e = lambda r, c, t=torch.bfloat16: torch.empty((r, c), dtype=t, device="cuda")      # noqa: E731
    for rows in (0, 64):
        dA, dB = sste.adapter_wgrad(e(rows, 72), e(rows, 64), e(rows, 8, torch.float32), e(rows, 8, torch.float32), rs, sa, 2,
                                    dA=torch.full((2, 8, 64), 3.0, device="cuda"), dB=torch.full((2, 8, 72), 3.0, device="cuda"))
        assert not dA.any() and not dB.any()
        dA, dB = sste.adapter_wgrad(e(rows, 72), e(rows, 64), e(rows, 8, torch.float32), e(rows, 8, torch.float32), rs, sa, 2,
                                    dA=torch.full((2, 8, 64), 3.0, device="cuda"), dB=torch.full((2, 8, 72), 3.0, device="cuda"), accumulate=True)
        assert (dA == 3).all() and (dB == 3).all()
    dA, dB = sste.adapter_wgrad(e(64, 0), e(64, 0), e(64, 8, torch.float32), e(64, 8, torch.float32), rs, sa, 2)
    assert dA.shape == (2, 8, 0) and dB.shape == (2, 8, 0)


@pytest.mark.parametrize("T", [64, 2300])
def test_wgrad_leaves_adapters_without_rows(sste, T):
    """accumulate: what an adapter without rows has stays as it is, bit for bit (negative zeros, NaN)."""
    rng = np.random.default_rng(8)
    X, dZ, S = normal(rng, (T, 64), 1).to(torch.bfloat16), normal(rng, (T, 72), 1).to(torch.bfloat16), normal(rng, (T, 16), 1)
    dA, dB = normal(rng, (40, 16, 64), 1), normal(rng, (40, 16, 72), 1)
    dA[3], dB[3], dA[39] = -0.0, float("nan"), -0.0
    kept = dA.clone(), dB.clone()
    sste.adapter_wgrad(dZ, X, S, S, *segments([0, 9, 30, 30, T - 2], [5, -1, 3, 7]), 40, dA=dA, dB=dB, accumulate=True)
    for got, want in zip((dA, dB), kept):
        same = (got.view(torch.int32) == want.view(torch.int32)).flatten(1)
        assert not same[5].all() and not same[7].all()
        same[[5, 7]] = True
        assert same.all()


def test_same_bits_every_time(sste):
    rng = np.random.default_rng(7)
    T = 9000
    X, dZ = normal(rng, (T, 264), 1).to(torch.bfloat16), normal(rng, (T, 136), 1).to(torch.bfloat16)
    S, dS = normal(rng, (T, 32), 1), normal(rng, (T, 32), 1)
    seg = segments([0, 3000, 5000, T], [1, 0, 1])
    first = sste.adapter_wgrad(dZ, X, S, dS, *seg, 2)
    for _ in range(3):
        again = sste.adapter_wgrad(dZ, X, S, dS, *seg, 2)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_native_marshalling(sste):
    """The same bits as through the Python definitions, outputs given or made; and the same refusals."""
    from paper_2409_09099_amd import binding
    rng = np.random.default_rng(17)
    T, I, O, R, N = 70, 144, 272, 16, 3
    X, dZ, A, B = (normal(rng, s, 1).to(torch.bfloat16) for s in ((T, I), (T, O), (N, R, I), (N, R, O)))
    scale, base = normal(rng, (N,), 1), normal(rng, (T, O), 1).to(torch.bfloat16)
    seg = segments([0, 30, 70], [2, 0])
    codes, blocks = sste.checkpoint_pack(X)
    S = normal(rng, (T, R), 1)
    X8 = (X.float() / 4).to(torch.float8_e4m3fn)
    wide = torch.empty((T, O + 8), dtype=torch.bfloat16, device="cuda")
    calls = [
        ("adapter_fwd", (X, *seg, A, B), {}), ("adapter_fwd", (X, *seg, A, B, scale, base), dict(Z=wide[:, :O], S=torch.empty_like(S))),
        ("adapter_fwd", (X8, *seg, A, B), dict(dtype=sste.F8E4M3, x_scale=4)), ("adapter_dgrad", (dZ, *seg, A, B), dict(scale=scale)),
        ("adapter_wgrad", (dZ, X, S, S, *seg, N), {}), ("adapter_wgrad", (dZ, codes, S, S, *seg, N), dict(x_dtype=sste.F8BLOCK, x_blocks=blocks)),
        ("adapter_wgrad", (dZ, X, S, S, *seg, N), dict(dA=torch.zeros((N, R, I), device="cuda"), dB=torch.zeros((N, R, O), device="cuda"), accumulate=True)),
        ("checkpoint_pack", (X,), {}), ("checkpoint_backward", (codes, blocks), {}), ("checkpoint_backward", (codes, blocks, X), dict(act=sste.ACT_NONE, restore=False)),
        ("checkpoint_backward", (codes, blocks, X), dict(A=torch.empty_like(X), dH=torch.empty_like(X))),
    ]
    for name, args, kw in calls:
        results = []
        for f in (binding._PYTHON[name], getattr(sste, name)):
            for k in ("dA", "dB"):
                if k in kw:
                    kw[k].fill_(0.5)
            results.append([None if t is None else t.clone() for t in f(*args, **kw)])
        assert [t is None for t in results[0]] == [t is None for t in results[1]]
        assert all(a is None or (a.dtype == b.dtype and torch.equal(a.view(torch.uint8) if a.is_contiguous() else a, b.view(torch.uint8) if b.is_contiguous() else b))
                   for a, b in zip(*results)), (name, kw.keys())
    i32 = torch.int32
    for call in (lambda: sste.adapter_fwd(X, seg[0].long(), seg[1], A, B), lambda: sste.adapter_fwd(X, seg[0], seg[1][:1], A, B), lambda: sste.adapter_fwd(X, *seg, A, B[:2]),
                 lambda: sste.adapter_fwd(X, *seg, A[:, :8], B), lambda: sste.adapter_fwd(X, *seg, B, A), lambda: sste.adapter_fwd(X, *seg, A, B, scale=scale[:2]),
                 lambda: sste.adapter_fwd(X, *seg, A, B, base=base[:9]), lambda: sste.adapter_fwd(X, *seg, A, B, Z=base.float()), lambda: sste.adapter_fwd(X, *seg, A, B, S=S[:, :8]),
                 lambda: sste.adapter_fwd(X, *seg, A.transpose(0, 1).contiguous().transpose(0, 1), B), lambda: sste.adapter_fwd(X.t(), *seg, A, B),
                 lambda: sste.adapter_dgrad(X, *seg, A, B), lambda: sste.adapter_wgrad(dZ[:9], X, S, S, *seg, N), lambda: sste.adapter_wgrad(dZ, X, S, S[:, :8], *seg, N),
                 lambda: sste.adapter_wgrad(dZ, X, S, S, *seg, N, accumulate=True), lambda: sste.adapter_wgrad(dZ, codes, S, S, *seg, N, x_dtype=sste.F8BLOCK),
                 lambda: sste.adapter_wgrad(dZ, X, S, S, *seg, N, dA=torch.zeros((N, R, I + 8), device="cuda")),
                 lambda: sste.adapter_fwd(X[:1].expand(T, I), *seg, A, B), lambda: sste.adapter_fwd(X, *seg, A[:, :1].expand(N, R, I), B), lambda: sste.adapter_fwd(X, *seg, A[:1].expand(N, R, I), B),
                 lambda: sste.adapter_fwd(X, *seg, A, B, base=base[:1].expand(T, O)), lambda: sste.adapter_wgrad(dZ[:1].expand(T, O), X, S, S, *seg, N), lambda: sste.checkpoint_pack(X[:1].expand(T, I)),
                 lambda: sste.adapter_fwd(X, *seg, A, B, workspace=codes[:1, :1].expand(1 << 20, 1)), lambda: sste.adapter_wgrad(dZ, X, S, S, *seg, N, workspace=codes[:1, :1].expand(1 << 20, 1)),
                 lambda: sste.checkpoint_pack(X, codes=codes[:9]), lambda: sste.checkpoint_pack(X, scales=torch.empty((T, 4), dtype=i32, device="cuda")),
                 lambda: sste.checkpoint_backward(codes, blocks[:, :2]), lambda: sste.checkpoint_backward(codes, blocks, dH=X), lambda: sste.checkpoint_backward(codes, blocks, A=X, restore=False)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sste.adapter_fwd(X, *seg, A[:, :, :], B, dtype=9), lambda: sste.checkpoint_backward(codes, blocks, act=7),
                 lambda: sste.adapter_wgrad(*(torch.zeros((4000, t.shape[1]), dtype=t.dtype, device="cuda") for t in (dZ, X, S, S)), *seg, N,
                                            workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(sste.SsteError):
            call()


# ---- together, streams, graphs --------------------------------------------------------------------------------------
def test_gradients_against_differences(sste):
    """The three calls chained as a layer's step are the gradient of sum(Z dZ) in X, A and B: against differences of the float64 forward pass."""
    rng = np.random.default_rng(9)
    T, I, O, R, N = 50, 64, 72, 8, 2
    X, dZ = normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (T, O), 1).to(torch.bfloat16)
    A, B, scale = normal(rng, (N, R, I), 0.1).to(torch.bfloat16), normal(rng, (N, R, O), 0.1).to(torch.bfloat16), torch.tensor([0.5, 2.0], device="cuda")
    starts, ids = [0, 20, 30, 45], [1, 0, 1]
    seg = segments(starts, ids)
    _, S = sste.adapter_fwd(X, *seg, A, B, scale=scale)
    dX, dS = sste.adapter_dgrad(dZ, *seg, A, B, scale=scale)
    dA, dB = sste.adapter_wgrad(dZ, X, S, dS, *seg, N)
    rows = OA.rows_of(starts, ids, N, T)
    v = {"X": f64(X), "A": f64(A), "B": f64(B)}
    loss = lambda: float((OA.apply(v["X"], rows, v["A"], v["B"], f64(scale), None)[0] * f64(dZ)).sum())      # noqa: E731
    # dA, dB: sums of up to 45 products, sum |products| at most a few times max |g|: 2^-17 of the split, 100 x 2^-23 of each of two accumulations
    for name, grad, step in (("X", dX, BF16_STEP), ("A", dA, 2.0 ** -14), ("B", dB, 2.0 ** -14)):
        g = f64(grad)
        for _ in range(6):
            at = tuple(rng.integers(0, n) for n in g.shape)
            kept = v[name][at]
            v[name][at] = kept + 0.5                                   # the loss is linear in each element: any difference will do
            up = loss()
            v[name][at] = kept - 0.5
            down = loss()
            v[name][at] = kept
            assert abs((up - down) - g[at]) <= step * np.abs(g).max() + 1e-9 * abs(up), (name, at)


@pytest.mark.parametrize("T,I,O,R", [(300, 136, 264, 16), (700, 2056, 520, 64), (2500, 2056, 520, 128)])          # one launch a product; shared out, with workspaces of the graph's own
def test_other_stream_and_graph(sste, T, I, O, R):
    """Captured once, replayed with other segments, adapters and rows written into the same tensors, between eager work."""
    rng = np.random.default_rng(11)
    N = 4
    X, dZ, base = (normal(rng, (T, n), 1).to(torch.bfloat16) for n in (I, O, O))
    A, B = normal(rng, (N, R, I), 0.1).to(torch.bfloat16), normal(rng, (N, R, O), 0.1).to(torch.bfloat16)
    rs, sa = segments([0, 100, 200, 300], [0, 1, 2])
    out = {k: torch.empty(s, dtype=d, device="cuda") for k, s, d in (("Z", (T, O), torch.bfloat16), ("S", (T, R), torch.float32), ("dX", (T, I), torch.bfloat16),
                                                                    ("dS", (T, R), torch.float32), ("dA", (N, R, I), torch.float32), ("dB", (N, R, O), torch.float32))}
    ws = torch.empty(sste.adapter_wgrad_workspace_bytes(T, 3, R, I, O), dtype=torch.uint8, device="cuda")

    def step():
        sste.adapter_fwd(X, rs, sa, A, B, base=base, Z=out["Z"], S=out["S"])
        sste.adapter_dgrad(dZ, rs, sa, A, B, dX=out["dX"], dS=out["dS"])
        sste.adapter_wgrad(dZ, X, out["S"], out["dS"], rs, sa, N, dA=out["dA"], dB=out["dB"], workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, (starts, ids) in enumerate([([0, 100, 200, 300], [0, 1, 2]), ([7, 7, 40, 290], [3, 3, 0]), ([0, 300, 300, 300], [2, 0, 1]), ([0, 10, 20, 30], [-1, 5, 1])]):
        rs.copy_(torch.tensor(starts, dtype=torch.int32))
        sa.copy_(torch.tensor(ids, dtype=torch.int32))
        X.copy_(normal(rng, (T, I), 1))
        step()
        want = {n: t.clone() for n, t in out.items()}
        for t in out.values():
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], want[n]), (k, n)


def test_two_streams_at_once(sste):
    """Two batches on two streams, each with its own workspaces and outputs, the same adapters: as one after the other."""
    rng = np.random.default_rng(29)
    T, I, O, R, N = 2500, 2056, 520, 128, 3
    A, B = normal(rng, (N, R, I), 0.1).to(torch.bfloat16), normal(rng, (N, R, O), 0.1).to(torch.bfloat16)
    batches = [(normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (T, O), 1).to(torch.bfloat16), *segments([0, n, T - 9], [2, k])) for n, k in ((700, 0), (33, 2))]

    def step(X, dZ, rs, sa):
        Z, S = sste.adapter_fwd(X, rs, sa, A, B)
        dX, dS = sste.adapter_dgrad(dZ, rs, sa, A, B)
        return (Z, S, dX, dS, *sste.adapter_wgrad(dZ, X, S, dS, rs, sa, N))

    want = [step(*b) for b in batches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    got = [[], []]
    for _ in range(10):
        for k, (stream, b) in enumerate(zip(streams, batches)):
            with torch.cuda.stream(stream):
                got[k].append(step(*b))
    torch.cuda.synchronize()
    for k in range(2):
        for results in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(results, want[k]))


def test_layer_with_adapters(sste):
    """A 2:4 layer in fine-tuning: projection, adapters on its output, both parts of the input gradient, the adapters' gradients from the layer's
    checkpointed input.  The whole output against the float64 layer."""
    from oracle import formats as F
    from oracle import projection as OP
    rng = np.random.default_rng(13)
    T, I, O, R, N = 192, 256, 320, 16, 2
    W, X, dZ = normal(rng, (O, I), 0.02).to(torch.bfloat16), normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (T, O), 1e-3).to(torch.bfloat16)
    A, B, scale = normal(rng, (N, R, I), 0.02).to(torch.bfloat16), normal(rng, (N, R, O), 0.02).to(torch.bfloat16), torch.tensor([2.0, 0.5], device="cuda")
    beta = np.float32(1.4830322)
    starts, ids = [0, 60, 130, 180], [1, 0, 1]
    seg = segments(starts, ids)
    vals, meta = sste.project_pack(W, float(beta))
    Z = sste.linear_fwd(X, vals, meta, O)
    sste.adapter_fwd(X, *seg, A, B, scale=scale, base=Z.clone(), Z=Z, S=(S := torch.empty((T, R), device="cuda")))
    codes, scales = sste.checkpoint_pack(X)
    dX = sste.linear_dgrad(dZ, vals, meta, I)
    _, dS = sste.adapter_dgrad(dZ, *seg, A, B, scale=scale, base=dX, dX=dX)
    dA, dB = sste.adapter_wgrad(dZ, codes, S, dS, *seg, N, x_dtype=sste.F8BLOCK, x_blocks=scales)
    torch.cuda.synchronize()
    rv, rm, _ = OP.project_pack(W.cpu().view(torch.int16).numpy().view(np.uint16), beta)
    dense = F.bf16_to_f32(rv).astype(np.float64)
    Wd = np.zeros((O, I))
    pos = np.stack([(rm & 3), (rm >> 2) & 3, (rm >> 4) & 3, (rm >> 6) & 3], axis=-1).reshape(O, I // 4, 2)
    np.put_along_axis(Wd.reshape(O, I // 4, 4), pos.astype(np.int64), dense.reshape(O, I // 4, 2), axis=2)
    rows = OA.rows_of(starts, ids, N, T)
    shared, back = f64(X) @ Wd.T, f64(dZ) @ Wd
    want, S64, _, eO = OA.apply(f64(X), rows, f64(A), f64(B), f64(scale), shared)
    # two roundings to bf16, the projection's output and the sum, and the projection's float32 accumulation
    slack = (I + 16) * OA.ACCUMULATE * (np.abs(f64(X)) @ np.abs(Wd).T)
    within("Z", Z, want, 1.01 * (eO + slack + BF16_STEP * (np.abs(shared) + np.abs(want))))
    want, dS64, _, eO = OA.apply(f64(dZ), rows, f64(B), f64(A), f64(scale), back)
    slack = (O + 16) * OA.ACCUMULATE * (np.abs(f64(dZ)) @ np.abs(Wd))
    within("dX", dX, want, 1.01 * (eO + slack + BF16_STEP * (np.abs(back) + np.abs(want))))
    x8 = OC.decode(codes.cpu().numpy(), scales.cpu().numpy())
    assert np.abs(x8 - f64(X)).max() <= 2.0 ** -4 * np.abs(f64(X)).max()
    for name, got, (G, e) in (("dA", dA, OA.outer(f64(dS), x8, rows, N)), ("dB", dB, OA.outer(f64(S), f64(dZ), rows, N))):
        within(name, got, G, e + 2.0 ** -22 * np.abs(G))
