"""The adapters' weight gradients of batches in many segments: their workspace and work go by the adapters, not by how the rows are cut."""
import numpy as np
import pytest
import torch

import paper_2409_09099_amd as sste
from oracle import adapter as OA
from oracle import checkpoint as OC


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


# ---- on the CPU: the workspace --------------------------------------------------------------------------------------
def test_workspace_by_adapters():
    size = sste.adapter_wgrad_workspace_bytes
    for segments in (7, 8, 64, 256):
        assert size(256, segments, 128, 1280, 5120, 1) == 0              # one adapter's rows, however they are cut
    assert size(256, 64, 128, 1280, 5120, 64) == 256 * 4 and size(256, 64, 128, 1280, 5120, 65) == size(256, 64, 128, 1280, 5120) > 64 * 128 * 6400 * 4
    table = 2048 * 4
    assert size(2048, 2048, 128, 1280, 5120, 8) == table                 # one block of rows: the table alone
    for segments in (1024, 16384):                                       # eight blocks: a sum for each adapter of each, the table and the adapters' rows
        assert size(16384, segments, 16, 4096, 4096, 4) == (8 * 4 * 16 * 8192 + 16384 + 8 * 4) * 4
    assert size(16384, 8, 16, 4096, 4096, 4) == size(16384, 8, 16, 4096, 4096)
    assert size(0, 300, 16, 64, 64, 3) == 0


def test_workspace_of_every_size():
    """Never more than without the number of adapters, and as many bytes as the ways of summing say."""
    for T in (0, 1, 255, 256, 2048, 2049, 5000, 40000, (1 << 27) - 1):
        for segments in (0, 1, 2, 256, 257, 700, 5000, 1 << 20):
            for adapters in (0, 1, 3, 300, 65535):
                for R in (8, 64, 128):
                    for a in (0, 8, 1280, 1 << 23):
                        for b in (0, 8, 5120, 1 << 23):
                            most, need = sste.adapter_wgrad_workspace_bytes(T, segments, R, a, b), sste.adapter_wgrad_workspace_bytes(T, segments, R, a, b, adapters)
                            assert need <= most, (T, segments, adapters, R, a, b)
                            if need != most:
                                blocks = -(-T // 2048)
                                sums = blocks * adapters if blocks > 1 else 0
                                assert need in (0, (-(-(T + sums) // 4) * 4 + sums * R * (a + b)) * 4), (T, segments, adapters, R, a, b)


def test_workspace_refusals():
    f, err = sste.library().sste_adapter_wgrad_workspace_bytes_ex, sste.library().sste_last_error
    for args in ((-1, 3, 2, 16, 64, 64), (4, -1, 2, 16, 64, 64), (4, 1, -1, 16, 64, 64), (4, 1, 65536, 16, 64, 64), (4, 1, 2, 15, 64, 64), (4, 1, 2, 16, 60, 64), (1 << 27, 1, 2, 16, 64, 64),
                 (4, (1 << 20) + 1, 2, 16, 64, 64), (1 << 62,) * 6):
        assert f(*args) == 0 and err().startswith(b"adapter_wgrad_workspace_bytes_ex: "), args
    assert f(300, 300, 2, 16, 64, 64) > 0 and err() == b""


# ---- on the GPU -----------------------------------------------------------------------------------------------------
def cut(T, segments, adapters, seed, bare=0.1):
    """Ragged segments, empty ones among them, rows before the first and behind the last, and some without an adapter or with one that there is not."""
    rng = np.random.default_rng(seed)
    starts = np.sort(rng.integers(min(T // 10, 3), T - T // 20 + 1, segments + 1)) if segments != T else np.arange(T + 1)
    ids = rng.integers(0, adapters, len(starts) - 1)
    ids[rng.random(len(ids)) < bare] = -1
    ids[rng.random(len(ids)) < 0.02] = adapters
    return starts.tolist(), ids.tolist()


def stored(t, kind):
    """(tensor, its float64 values, format, scale, scales of blocks)"""
    if kind == "bf16":
        t = t.to(torch.bfloat16)
        return t, f64(t), sste.BF16, 1.0, None
    if kind == "checkpoint":
        codes, blocks = sste.checkpoint_pack(t.to(torch.bfloat16))
        return codes, OC.decode(codes.cpu().numpy(), blocks.cpu().numpy()), sste.F8BLOCK, 1.0, blocks
    dtype = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[kind]
    scale = float(t.abs().max()) / torch.finfo(dtype).max
    t = (t / scale).to(dtype)
    return t, f64(t) * float(np.float32(scale)), {"e4m3": sste.F8E4M3, "e5m2": sste.F8E5M2}[kind], scale, None


def launches(call):
    sste.timing_begin(64)
    try:
        result = call()
    finally:
        times = sste.timing_end()
    return result, times["adapter"][1]


def check(T, I, O, R, adapters, starts, ids, count, kind="bf16", x_kind="bf16", accumulate=False, pad=0, seed=0):
    rng = np.random.default_rng(seed)
    normal = lambda *shape, std=1.0: torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).cuda()      # noqa: E731

    def room(t):
        """The rows of a wider matrix with something else behind them."""
        r = torch.full((t.shape[0], t.shape[1] + pad), 77, device="cuda").to(t.dtype) if t.dtype != torch.float32 else torch.full((t.shape[0], t.shape[1] + pad), float("nan"), device="cuda")
        r[:, :t.shape[1]] = t
        return r[:, :t.shape[1]] if pad else t

    dZ, dz64, dt, dzs, _ = stored(normal(T, O, std=1e-3), kind)
    X, x64, xdt, xs, blocks = stored(normal(T, I), x_kind)
    rows = OA.rows_of(starts, ids, adapters, T)
    S, dS = normal(T, R), normal(T, R, std=1e-3)
    s64, ds64 = np.where(rows[:, None] < 0, 0, f64(S)), f64(dS)
    S[torch.from_numpy(rows < 0).cuda()] = float("nan")                   # not read where there is no adapter
    dA, dB, kept = None, None, [0.0, 0.0]
    if accumulate or pad:
        dA, dB = (torch.empty((adapters, R, w + pad), device="cuda")[:, :, :w].copy_(normal(adapters, R, w)) for w in (I, O))
    if accumulate:
        kept = [f64(dA), f64(dB)]
    row_start, seg = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (starts, ids))
    call = lambda: sste.adapter_wgrad(room(dZ), room(X), room(S), room(dS), row_start, seg, adapters, dtype=dt, dy_scale=dzs, x_dtype=xdt, x_scale=xs, x_blocks=blocks, dA=dA, dB=dB,      # noqa: E731
                                      accumulate=accumulate)
    (dA, dB), number = launches(call)
    assert number == count
    for name, got, (want, bound), old in (("dA", dA, OA.outer(ds64, x64, rows, adapters), kept[0]), ("dB", dB, OA.outer(s64, dz64, rows, adapters), kept[1])):
        # The bound counts 3 n + 8 additions for an adapter of n rows; the sum of b blocks' sums is b - 1 more for a row than its own block has, which has at least
        # b - 1 rows less.  Two for scale and what was there.
        err, limit = np.abs(f64(got) - (want + old)), bound + OA.ACCUMULATE * (np.abs(want) + np.abs(old)) * 2
        assert (err <= limit).all(), (name, err.max(), np.argwhere(~(err <= limit))[:4])
        for n in set(range(adapters)) - set(rows.tolist()):
            assert np.array_equal(f64(got[n]), old[n] if accumulate else np.zeros_like(want[n]))


FEW, BLOCK, CHUNKS, BLOCKS = 1, 2, 2, 3          # launches: few segments' rows; one block of rows with its table; chunks and their sums; several blocks with a table and their sum
CASES = [
    (256, 1280, 520, 128, 1, 64, FEW), (256, 264, 136, 128, 3, 256, FEW), (2000, 136, 72, 96, 2, 200, FEW), (1, 64, 72, 8, 1, 1, FEW),
    (256, 136, 72, 24, 5, 257, BLOCK), (300, 8, 520, 8, 150, 300, BLOCK), (2047, 128, 264, 40, 3, 2047, BLOCK), (2048, 136, 128, 16, 7, 1000, BLOCK), (90, 264, 0, 64, 2, 4000, BLOCK),
    (3000, 136, 264, 40, 60, 100, CHUNKS), (1000, 72, 136, 16, 301, 300, CHUNKS), (9000, 136, 72, 24, 9, 70, CHUNKS),
    (2049, 136, 264, 24, 3, 300, BLOCKS), (4096, 72, 136, 64, 9, 400, BLOCKS), (4097, 1032, 144, 16, 20, 4097, BLOCKS), (9000, 208, 400, 128, 4, 1500, BLOCKS), (5000, 0, 136, 8, 600, 5000, BLOCKS),
]


@pytest.mark.gpu
@pytest.mark.parametrize("T,I,O,R,adapters,segments,count", CASES)
def test_many_segments(T, I, O, R, adapters, segments, count):
    check(T, I, O, R, adapters, *cut(T, segments, adapters, T + R), count)


@pytest.mark.gpu
@pytest.mark.parametrize("T,segments,count", [(333, 300, BLOCK), (2333, 400, BLOCKS)])
@pytest.mark.parametrize("kind,x_kind", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e5m2", "checkpoint"), ("bf16", "checkpoint"), ("bf16", "bf16")])
@pytest.mark.parametrize("R", [8, 32, 64, 128])
def test_formats(kind, x_kind, R, T, segments, count):
    check(T, 208, 400, R, 3, *cut(T, segments, 3, R), count, kind, x_kind)


@pytest.mark.gpu
@pytest.mark.parametrize("T,segments,count", [(200, 100, FEW), (500, 400, BLOCK), (2500, 400, BLOCKS)])
@pytest.mark.parametrize("accumulate,pad", [(True, 0), (True, 16), (False, 16)])
def test_accumulates_and_strides(accumulate, pad, T, segments, count):
    check(T, 144, 272, 16, 7, *cut(T, segments, 6, 5), count, accumulate=accumulate, pad=pad)


@pytest.mark.gpu
@pytest.mark.parametrize("T,segments,count", [(500, 400, BLOCK), (2500, 400, BLOCKS)])
def test_accumulate_leaves_adapters_without_rows(T, segments, count):
    rng = np.random.default_rng(8)
    normal = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()      # noqa: E731
    X, dZ, S, dA, dB = normal(T, 64).bfloat16(), normal(T, 72).bfloat16(), normal(T, 16), normal(40, 16, 64), normal(40, 16, 72)
    dA[3], dB[3], dA[39] = -0.0, float("nan"), -0.0
    kept = dA.clone(), dB.clone()
    rows = torch.linspace(0, T - 2, segments + 1).int().cuda(), torch.tensor([5, 7, -1, 40], dtype=torch.int32, device="cuda").repeat(segments // 4)
    _, number = launches(lambda: sste.adapter_wgrad(dZ, X, S, S, *rows, 40, dA=dA, dB=dB, accumulate=True))
    assert number == count
    for got, want in zip((dA, dB), kept):
        same = (got.view(torch.int32) == want.view(torch.int32)).flatten(1)
        assert not same[5].all() and not same[7].all()
        same[[5, 7]] = True
        assert same.all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,segments,count", [(500, 400, BLOCK), (2500, 400, BLOCKS)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_keeps_to_its_rows(T, segments, count, kind):
    """NaN in the rows of one adapter, of none and of no segment reach no other adapter's gradients."""
    rng = np.random.default_rng(6)
    normal = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()      # noqa: E731
    X, dZ, S, dS = normal(T, 144).to(torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn), normal(T, 80).bfloat16(), normal(T, 40), normal(T, 40)
    starts, ids = cut(T, segments, 3, 9, bare=0.2)
    seg = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (starts, ids)]
    dt = sste.BF16 if kind == "bf16" else sste.F8E4M3
    want, number = launches(lambda: sste.adapter_wgrad(dZ, X, S, dS, *seg, 3, x_dtype=dt))
    assert number == count
    hit = torch.from_numpy(np.isin(OA.rows_of(starts, ids, 3, T), (-1, 1))).cuda()
    for t in (dZ, S, dS):
        t[hit] = float("nan")
    X.view(torch.int16 if kind == "bf16" else torch.uint8)[hit] = 0x7FC0 if kind == "bf16" else 0x7F
    dA, dB = sste.adapter_wgrad(dZ, X, S, dS, *seg, 3, x_dtype=dt)
    for n in (0, 2):
        assert torch.equal(dA[n], want[0][n]) and torch.equal(dB[n], want[1][n])
    assert dA[1].isnan().all() and dB[1].isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,segments", [(100, 300), (2300, 300)])
def test_malformed_bounds_stay_inside(T, segments):
    """Bounds outside the rows, and bounds that decrease: what is written stays inside, and bounds beyond the ends mean the ends."""
    rng = np.random.default_rng(1)
    R, I, O, N = 16, 64, 72, 2
    normal = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()      # noqa: E731
    X, dZ, S = normal(T, I).bfloat16(), normal(T, O).bfloat16(), normal(T, R)
    ids = torch.from_numpy(rng.integers(-1, N, segments).astype(np.int32)).cuda()
    inside = np.sort(rng.integers(0, T + 1, segments + 1))
    inside[0], inside[-1] = 0, T
    outside = inside.copy()
    outside[0], outside[-1] = -2 ** 31, 2 ** 31 - 1
    need = sste.adapter_wgrad_workspace_bytes(T, segments, R, I, O, N)
    results = []
    for starts in (inside, outside, rng.integers(-T, 2 * T, segments + 1), inside[::-1].copy()):
        ws, room_a, room_b = torch.full((need + 256,), 0x11, dtype=torch.uint8, device="cuda"), torch.full((N + 2, R, I), 7.0, device="cuda"), torch.full((N + 2, R, O), 7.0, device="cuda")
        sste.adapter_wgrad(dZ, X, S, S, torch.from_numpy(starts.astype(np.int32)).cuda(), ids, N, dA=room_a[1:-1], dB=room_b[1:-1], workspace=ws[:need])
        assert (ws[need:] == 0x11).all() and all((r[0] == 7).all() and (r[-1] == 7).all() for r in (room_a, room_b))
        results.append((room_a, room_b))
    assert all(torch.equal(a, b) for a, b in zip(results[0], results[1]))


@pytest.mark.gpu
def test_workspaces():
    """What the query without the adapters asks for serves as well, with the same bits; less than the query with them asks for is refused."""
    rng = np.random.default_rng(3)
    T, R, I, O, N = 2500, 16, 64, 72, 3
    normal = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()      # noqa: E731
    args = normal(T, O).bfloat16(), normal(T, I).bfloat16(), normal(T, R), normal(T, R), *(torch.tensor(v, dtype=torch.int32, device="cuda") for v in cut(T, 500, N, 2)), N
    need, most = sste.adapter_wgrad_workspace_bytes(T, 500, R, I, O, N), sste.adapter_wgrad_workspace_bytes(T, 500, R, I, O)
    assert 0 < need < most // 20
    want = sste.adapter_wgrad(*args)
    for size in (need, most):
        got = sste.adapter_wgrad(*args, workspace=torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda"))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(sste.SsteError):
        sste.adapter_wgrad(*args, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [500, 2500])
def test_graph(T):
    """Captured once, replayed with other bounds and adapters, between eager work."""
    rng = np.random.default_rng(11)
    R, I, O, N, segments = 24, 136, 264, 4, 400
    normal = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()      # noqa: E731
    X, dZ, S, dS = normal(T, I).bfloat16(), normal(T, O).bfloat16(), normal(T, R), normal(T, R)
    rs, sa = torch.zeros(segments + 1, dtype=torch.int32, device="cuda"), torch.zeros(segments, dtype=torch.int32, device="cuda")
    dA, dB = torch.empty((N, R, I), device="cuda"), torch.empty((N, R, O), device="cuda")
    step = lambda: sste.adapter_wgrad(dZ, X, S, dS, rs, sa, N, dA=dA, dB=dB)      # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        starts, ids = cut(T, segments, N - 1 if k == 2 else N, 20 + k)
        rs.copy_(torch.tensor(starts, dtype=torch.int32))
        sa.copy_(torch.tensor(ids, dtype=torch.int32))
        X.copy_(normal(T, I))
        step()
        want = dA.clone(), dB.clone()
        dA.fill_(float("nan"))
        dB.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dA, want[0]) and torch.equal(dB, want[1]), k
