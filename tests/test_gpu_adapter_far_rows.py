"""Rows of the adapters' matrices that lie beyond 2^32 bytes: views of wide buffers, used in their first columns only, for each way of computing the calls."""
import numpy as np
import pytest
import torch

from test_gpu_adapter import normal, segments

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sste():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_09099_amd as lib
    lib.library()
    return lib


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e5m2"])
@pytest.mark.parametrize("shared", [True, False])
def test_far_rows_in_two_launches(sste, kind, shared):
    """Row offsets beyond 2^32 bytes in every matrix of both kernels."""
    T, K, C, R = 700, 2064, 136, 64
    ld, ldf = 1 << 23, 1 << 21                                            # bytes of a row, and floats of one: 700 rows are 5.9 GB
    rng = np.random.default_rng(3)
    x, base = normal(rng, (T, K), 1), normal(rng, (T, C), 1).to(torch.bfloat16)
    down, up = normal(rng, (2, R, K), 0.05).to(torch.bfloat16), normal(rng, (2, R, C), 0.05).to(torch.bfloat16)
    x = x.to({"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[kind])
    need = sste.adapter_workspace_bytes(T, 3, R, K, C)
    assert need > 0
    ws = torch.empty(need if shared else 0, dtype=torch.uint8, device="cuda")
    seg = segments([0, T // 2, T // 2 + 9, T - 7], [1, -1, 0])
    room, floats = torch.empty((T, ld), dtype=torch.uint8, device="cuda"), torch.empty((T, ldf), device="cuda")
    far_x = room.view(x.dtype)[:, :K]
    far_x.copy_(x) if kind == "bf16" else room[:, :K].copy_(x.view(torch.uint8))
    far_base, far_out, far_s = room.view(torch.bfloat16)[:, 1 << 20:(1 << 20) + C], room.view(torch.bfloat16)[:, 1 << 21:(1 << 21) + C], floats[:, :R]
    far_base.copy_(base)
    dtype = {"bf16": sste.BF16, "e4m3": sste.F8E4M3, "e5m2": sste.F8E5M2}[kind]
    if kind == "e5m2":
        call = lambda x, base, **out: sste.adapter_dgrad(x, *seg, up, down, base=base, dtype=dtype, workspace=ws, **{{"Z": "dX", "S": "dS"}[k]: v for k, v in out.items()})      # noqa: E731
    else:
        call = lambda x, base, **out: sste.adapter_fwd(x, *seg, down, up, base=base, dtype=dtype, workspace=ws, **out)      # noqa: E731
    want = call(x, base)
    sste.timing_begin(16)
    try:
        call(far_x, far_base, Z=far_out, S=far_s)
    finally:
        times = sste.timing_end()
    assert times["adapter"][1] == 2
    assert torch.equal(far_out, want[0]) and torch.equal(far_s, want[1])


@pytest.mark.parametrize("T,count,ids", [(600, 1, 2), (600, 2, 400), (2100, 3, 400), (2100, 2, 2)])
def test_far_rows_of_the_weight_gradients(sste, T, count, ids):
    """Row offsets beyond 2^32 bytes in the operands and in S and dS, for each way of summing."""
    R, I, O = 16, 64, 80
    rng = np.random.default_rng(4)
    x, dz, s = normal(rng, (T, I), 1).to(torch.bfloat16), normal(rng, (T, O), 1).to(torch.bfloat16), normal(rng, (T, R), 1)
    room, floats = torch.empty((T, 1 << 22), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 1 << 21), device="cuda")
    room[:, :I], room[:, 128:128 + O], floats[:, :R], floats[:, 64:64 + R] = x, dz, s, 2 * s
    seg = segments(np.linspace(0, T - 3, ids + 1).astype(int).tolist(), [k % 2 for k in range(ids)])
    want = sste.adapter_wgrad(dz, x, s, 2 * s, *seg, 2)
    sste.timing_begin(16)
    try:
        got = sste.adapter_wgrad(room[:, 128:128 + O], room[:, :I], floats[:, :R], floats[:, 64:64 + R], *seg, 2)
    finally:
        times = sste.timing_end()
    assert times["adapter"][1] == count
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
