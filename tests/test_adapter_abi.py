"""Refusals of the adapter and checkpoint calls: the C ABI's status codes, and the binding's own checks (no GPU: nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2409_09099_amd as sste

P = ctypes.c_void_p
FAKE, ODD = P(0x1000), P(0x1004)      # never dereferenced: validation fails first
HUGE = 1 << 62


@pytest.fixture(scope="module")
def lib():
    return sste.library()


def err(lib):
    return lib.sste_last_error().decode()


# argument numbers: 0 X 1 T 2 I 3 ldx 4 dtype 5 x_scale 6 row_start 7 segments 8 seg_adapter 9 A 10 lda 11 B 12 ldb 13 scale 14 adapters 15 R 16 O 17 base 18 ldbase 19 Z 20 ldz
# 21 S 22 lds 23 workspace 24 bytes 25 stream
FWD = [FAKE, 4, 64, 64, 0, 1.0, FAKE, 2, FAKE, FAKE, 64, FAKE, 80, FAKE, 3, 16, 80, FAKE, 80, P(0x2000), 80, FAKE, 16, None, 0, None]


@pytest.mark.parametrize("change,status", [
    ({1: -1}, 2), ({7: -1}, 2), ({14: -1}, 2), ({2: -8}, 2), ({16: -8}, 2), ({15: 0}, 2), ({15: -8}, 2),
    ({15: 12}, 7), ({15: 136}, 7), ({2: 60, 3: 64}, 7), ({16: 76}, 7), ({2: 1 << 25, 3: 1 << 25, 10: 1 << 25}, 7), ({1: 1 << 27}, 7), ({7: (1 << 20) + 1}, 7), ({14: 65536}, 7),
    ({3: 56}, 2), ({10: 56}, 2), ({12: 72}, 2), ({18: 72}, 2), ({20: 72}, 2), ({22: 12}, 2),
    ({3: 68}, 3), ({10: 68}, 3), ({12: 84}, 3), ({18: 84}, 3), ({20: 84}, 3), ({22: 18}, 3),
    ({0: ODD}, 3), ({9: ODD}, 3), ({11: ODD}, 3), ({17: ODD}, 3), ({19: ODD}, 3), ({21: ODD}, 3), ({6: P(0x1002)}, 3), ({8: P(0x1001)}, 3), ({13: P(0x1002)}, 3),
    ({4: 2}, 4), ({4: 3}, 4), ({4: 4}, 4), ({4: 7}, 4),
    ({5: 0.0}, 5), ({5: -1.0}, 5), ({5: float("nan")}, 5), ({5: float("inf")}, 5), ({5: 2.0}, 5), ({17: P(0x2000), 18: 88}, 5),
    ({0: None}, 1), ({6: None}, 1), ({8: None}, 1), ({9: None}, 1), ({11: None}, 1), ({19: None}, 1), ({21: None}, 1),
    ({4: 1, 2: 72, 3: 80, 10: 72}, 7), ({4: 1, 2: 64, 3: 72}, 3),          # 8-bit rows are multiples of 16
    ({3: HUGE}, 7), ({20: HUGE}, 7), ({22: HUGE}, 7), ({10: HUGE}, 7),
    ({1: 2040, 7: 953, 16: 1 << 23, 12: 1 << 23, 18: 1 << 23, 20: 1 << 23}, 7),          # tiles that a grid, rounded up to the XCDs, cannot count
])
def test_adapter_fwd_refuses(lib, change, status):
    args = [change.get(i, v) for i, v in enumerate(FWD)]
    assert lib.sste_adapter_fwd(*args) == status and err(lib).startswith("adapter_fwd: ")


# 0 dZ 1 T 2 O 3 lddz 4 dtype 5 dz_scale ... 16 I: the same places, A as wide as dX and B as wide as dZ
DGRAD = [FAKE, 4, 80, 80, 3, 0.5, FAKE, 2, FAKE, FAKE, 64, FAKE, 80, FAKE, 3, 16, 64, FAKE, 64, P(0x2000), 64, FAKE, 16, None, 0, None]


@pytest.mark.parametrize("change,status", [({4: 2}, 4), ({4: 4}, 4), ({4: 0}, 5), ({12: 72}, 2), ({10: 56}, 2), ({2: 72, 12: 72}, 7), ({15: 9}, 7), ({20: 56}, 2), ({9: None}, 1), ({11: None}, 1)])
def test_adapter_dgrad_refuses(lib, change, status):
    args = [change.get(i, v) for i, v in enumerate(DGRAD)]
    assert lib.sste_adapter_dgrad(*args) == status and err(lib).startswith("adapter_dgrad: ")


# 0 dZ 1 T 2 O 3 lddz 4 dtype 5 dz_scale 6 X 7 I 8 ldx 9 x_dtype 10 x_scale 11 x_blocks 12 ldxb 13 S 14 lds 15 dS 16 ldds 17 row_start 18 segments 19 seg_adapter 20 adapters 21 R
# 22 dA 23 ldda 24 dB 25 lddb 26 accumulate 27 workspace 28 bytes 29 stream
WGRAD = [FAKE, 4000, 80, 80, 0, 1.0, FAKE, 64, 64, 0, 1.0, None, 0, FAKE, 16, FAKE, 16, FAKE, 2, FAKE, 3, 16, FAKE, 64, FAKE, 80, 0, FAKE, 1 << 40, None]


@pytest.mark.parametrize("change,status", [
    ({1: -1}, 2), ({2: -8}, 2), ({7: -8}, 2), ({18: -1}, 2), ({20: -1}, 2), ({21: 0}, 2), ({21: 20}, 7), ({2: 76}, 7), ({7: 60}, 7),
    ({3: 72}, 2), ({8: 56}, 2), ({14: 12}, 2), ({16: 12}, 2), ({23: 60}, 2), ({25: 76}, 2), ({9: 4, 11: FAKE, 12: 1}, 2),
    ({3: 84}, 3), ({8: 68}, 3), ({14: 18}, 3), ({23: 66}, 3), ({25: 82}, 3), ({0: ODD}, 3), ({6: ODD}, 3), ({13: ODD}, 3), ({15: ODD}, 3), ({22: ODD}, 3), ({24: ODD}, 3), ({27: ODD}, 3),
    ({4: 2}, 4), ({4: 4}, 4), ({9: 2}, 4), ({9: 3}, 4), ({5: 2.0}, 5), ({10: 2.0}, 5), ({9: 4, 10: 2.0, 11: FAKE, 12: 2}, 5), ({10: -1.0}, 5), ({26: 2}, 5),
    ({0: None}, 1), ({6: None}, 1), ({13: None}, 1), ({15: None}, 1), ({17: None}, 1), ({22: None}, 1), ({24: None}, 1), ({9: 4, 12: 2}, 1),
    ({27: None}, 6), ({28: 16}, 6), ({18: 1 << 20, 2: 1024, 3: 1024, 25: 1024, 7: 1024, 8: 1024, 23: 1024}, 7), ({8: HUGE}, 7), ({9: 4, 11: FAKE, 12: HUGE}, 7),
])
def test_adapter_wgrad_refuses(lib, change, status):
    args = [change.get(i, v) for i, v in enumerate(WGRAD)]
    assert lib.sste_adapter_wgrad(*args) == status and err(lib).startswith("adapter_wgrad: ")


def test_wgrad_workspace(lib):
    f = lib.sste_adapter_wgrad_workspace_bytes
    assert f(0, 3, 16, 64, 64) == 0
    assert f(256, 256, 16, 64, 128) == 0                                  # few rows: one launch without chunks
    for more in ((2049, 3), (100, 257)):
        need = f(*more, 16, 64, 128)
        assert need > 0 and need % (16 * 192 * 4) == 0
    assert f(-1, 3, 16, 64, 64) == 0 and f(4, -1, 16, 64, 64) == 0 and f(4, 1, 15, 64, 64) == 0 and f(4, 1, 16, 60, 64) == 0 and f(1 << 27, 1, 16, 64, 64) == 0
    args = list(WGRAD)
    args[28] = sste.adapter_wgrad_workspace_bytes(4000, 2, 16, 64, 80) - 1
    assert lib.sste_adapter_wgrad(*args) == 6


def test_plans_of_every_size(lib):
    """The planning of a call is host arithmetic: every combination of ends must come to a size, with nothing divided by zero on the way."""
    for T in (0, 1, 9, 15, 16, 17, 600, 5000, 9000, 40000, (1 << 27) - 1):
        for segments in (0, 1, 2, 700, 1 << 20):
            for R in (8, 16, 32, 64, 128):
                for a in (0, 8, 64, 5120, 1 << 23):
                    for b in (0, 8, 1280, 1 << 23):
                        need = lib.sste_adapter_workspace_bytes(T, segments, R, a, b)
                        assert (need == 0) if T == 0 else need % (T * R * 4) == 0 and need // (T * R * 4) in (0, 2, 3, 4), (T, segments, R, a, b)
                        need = lib.sste_adapter_wgrad_workspace_bytes(T, segments, R, a, b)
                        few = T <= 2048 and segments <= 256 and T * R * (a + b) * max(segments, 8) <= 6e9
                        assert (need == 0) == (few or T == 0 or a + b == 0) and (a + b == 0 or need % (R * (a + b) * 4) == 0)


@pytest.mark.parametrize("change,status", [({1: -1}, 2), ({2: -16}, 2), ({2: 24}, 7), ({1: 1 << 31}, 7), ({3: 32}, 2), ({3: 50}, 3), ({0: ODD}, 3), ({0: None}, 1), ({4: None}, 1), ({6: None}, 1),
                                            ({4: ODD}, 3), ({5: 32}, 2), ({5: 56}, 3), ({7: 1}, 2), ({3: HUGE}, 7), ({5: HUGE}, 7), ({7: HUGE}, 7)])
def test_checkpoint_pack_refuses(lib, change, status):
    args = [change.get(i, v) for i, v in enumerate([FAKE, 4, 48, 48, FAKE, 48, FAKE, 2, None])]
    assert lib.sste_checkpoint_pack(*args) == status and err(lib).startswith("checkpoint_pack: ")


# 0 codes 1 scales 2 R 3 C 4 ldc 5 lds 6 act 7 A 8 lda 9 dA 10 ldda 11 dH 12 lddh 13 stream
@pytest.mark.parametrize("change,status", [({2: -1}, 2), ({3: -16}, 2), ({3: 40}, 7), ({4: 32}, 2), ({4: 56}, 3), ({5: 1}, 2), ({6: 2}, 5), ({8: 40}, 2), ({8: 52}, 3), ({10: 40}, 2), ({12: 40}, 2),
                                            ({0: None}, 1), ({1: None}, 1), ({9: None}, 1), ({11: None}, 1), ({7: None, 9: None, 11: None}, 1), ({7: ODD}, 3), ({9: ODD}, 3), ({11: ODD}, 3),
                                            ({11: FAKE, 12: 56}, 5), ({12: HUGE}, 7)])
def test_checkpoint_backward_refuses(lib, change, status):
    args = [change.get(i, v) for i, v in enumerate([FAKE, FAKE, 4, 48, 48, 2, 1, FAKE, 48, FAKE, 48, P(0x2000), 48, None])]
    assert lib.sste_checkpoint_backward(*args) == status and err(lib).startswith("checkpoint_backward: ")


def test_nothing_to_do_is_no_error(lib):
    """No rows: accepted without a launch (there is no GPU here)."""
    args = list(FWD)
    args[1] = 0
    for i in (0, 17, 19, 21):
        args[i] = None
    assert lib.sste_adapter_fwd(*args) == 0
    assert lib.sste_checkpoint_pack(None, 0, 48, 48, None, 48, None, 2, None) == 0
    assert lib.sste_checkpoint_pack(None, 4, 0, 0, None, 0, None, 0, None) == 0
    assert lib.sste_checkpoint_backward(None, None, 0, 48, 48, 2, 1, None, 48, None, 48, None, 48, None) == 0


def test_binding_refuses():
    """What the binding checks before the library is asked; tensors on the CPU are the last of it."""
    z = lambda *n, t=torch.bfloat16: torch.zeros(n, dtype=t)      # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32)             # noqa: E731
    for call in (lambda: sste.adapter_fwd(z(4, 64), i(0, 4), i(0), z(1, 8, 64), z(1, 8, 80)),
                 lambda: sste.adapter_dgrad(z(4, 80), i(0, 4), i(0), z(1, 8, 64), z(1, 8, 80)),
                 lambda: sste.adapter_wgrad(z(4, 80), z(4, 64), z(4, 8, t=torch.float32), z(4, 8, t=torch.float32), i(0, 4), i(0), 1),
                 lambda: sste.checkpoint_pack(z(4, 64)),
                 lambda: sste.checkpoint_backward(z(4, 64, t=torch.uint8), z(4, 2, t=torch.uint8)),
                 lambda: sste.adapter_fwd(z(4), i(0, 4), i(0), z(1, 8, 64), z(1, 8, 80))):
        with pytest.raises(ValueError):
            call()


def test_binding_refuses_overlapping_rows():
    """Rows that share memory (an expanded tensor) have no leading dimension; told by shape and strides alone."""
    from types import SimpleNamespace
    from paper_2409_09099_amd import binding
    like = lambda shape, strides: SimpleNamespace(dim=lambda: len(shape), is_cuda=True, element_size=lambda: 2, shape=shape, stride=lambda i: strides[i])      # noqa: E731
    for strides in ((0, 1), (63, 1), (8, 1)):
        with pytest.raises(ValueError):
            binding._matrix(like((4, 64), strides), 2, "X")
    assert binding._matrix(like((4, 64), (64, 1)), 2, "X") == (4, 64, 64) and binding._matrix(like((1, 64), (0, 1)), 2, "X") == (1, 64, 64)
    assert binding._matrix(like((0, 64), (0, 1)), 2, "X") == (0, 64, 64) and binding._matrix(like((4, 0), (1, 1)), 2, "X")[:2] == (4, 0)
