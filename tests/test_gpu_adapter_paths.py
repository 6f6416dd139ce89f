"""Every form of the adapters' kernels that a size can lead to: one launch or two, tiles of 32 or 64 rows, the contraction shared out or not, each operand
format and rank.  The number of launches and of parts is asserted, so that a change of the choice between them cannot leave a form without a test."""
import pytest
import torch

from test_gpu_adapter import check_apply

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sste():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2409_09099_amd as lib
    lib.library()
    return lib


# rows, width in, width out, rank, launches, parts of the contraction; in the comment the rows of a tile of the first product
PATHS = [
    (300, 272, 136, 16, 1, 0), (300, 272, 136, 32, 1, 0), (300, 272, 136, 64, 1, 0), (300, 272, 136, 128, 1, 0), (4100, 2576, 1032, 32, 1, 0),                    # 16
    (16000, 272, 136, 16, 2, 0), (3000, 5120, 1032, 16, 2, 4),                                                                        # 32
    (300, 5120, 136, 32, 2, 4),                                                                                                       # 32
    (16000, 272, 136, 32, 2, 0), (3000, 5120, 1032, 32, 2, 4),                                          # 64
    (6500, 1040, 136, 64, 2, 0), (300, 2064, 136, 64, 2, 4),                                                                          # 32
    (9000, 272, 136, 64, 2, 0), (6500, 2064, 136, 64, 2, 2), (5003, 2064, 136, 64, 2, 3),                                             # 64
    (4100, 272, 136, 128, 2, 0), (300, 1040, 136, 128, 2, 4),                                                                         # 32
    (9000, 272, 136, 128, 2, 0), (6500, 1040, 136, 128, 2, 2), (4100, 1040, 136, 128, 2, 3),                                          # 64
]


@pytest.mark.parametrize("T,K,C,R,count,parts", PATHS)
@pytest.mark.parametrize("fwd,kind", [(True, "bf16"), (True, "e4m3"), (False, "e4m3"), (False, "e5m2")])
def test_every_form(sste, T, K, C, R, count, parts, fwd, kind):
    starts, ids = [5, 70, 134, 199, T - 20], [2, -1, 0, 1]
    assert sste.adapter_workspace_bytes(T, len(ids), R, K, C) == parts * T * R * 4
    sste.timing_begin(16)
    try:
        check_apply(sste, fwd, T, K, C, R, 3, starts, ids, kind, seed=R)
    finally:
        times = sste.timing_end()
    assert times["adapter"][1] == count


@pytest.mark.parametrize("T,K,C,R", [p[:4] for p in PATHS if p[5] > 1])
@pytest.mark.parametrize("fwd,kind", [(True, "e4m3"), (False, "e5m2")])
def test_contraction_not_shared_out(sste, T, K, C, R, fwd, kind):
    """Without room for the parts' sums."""
    need = sste.adapter_workspace_bytes(T, 4, R, K, C)
    for size in (0, need - 1):
        check_apply(sste, fwd, T, K, C, R, 3, [5, 70, 134, 199, T - 20], [2, -1, 0, 1], kind, workspace=torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda"), seed=R)
