"""What the matrices of the adapter and checkpoint calls may be kept in: the format's own type or its raw bits.  Another floating-point type of the same
width would be read as if it were the format, with no sign of it in the result."""
from types import SimpleNamespace

import pytest
import torch

import paper_2409_09099_amd as sste
from paper_2409_09099_amd import binding

RAW = {2: (torch.int16, torch.uint16), 1: (torch.uint8, torch.int8)}
OWN = {sste.BF16: torch.bfloat16, sste.F8E4M3: torch.float8_e4m3fn, sste.F8E5M2: torch.float8_e5m2, sste.F8BLOCK: torch.float8_e4m3fn}
ALL = (torch.float16, torch.bfloat16, torch.int16, torch.uint16, torch.bool, torch.uint8, torch.int8, torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz)


@pytest.mark.parametrize("kind", list(OWN))
@pytest.mark.parametrize("dtype", ALL, ids=str)
def test_types_of_each_format(kind, dtype):
    tensor = SimpleNamespace(dtype=dtype)
    if dtype == OWN[kind] or dtype in RAW[OWN[kind].itemsize]:
        binding._holds(tensor, kind, "X")
    else:
        with pytest.raises(ValueError, match="X must be .* not " + str(dtype)):
            binding._holds(tensor, kind, "X")


def arguments():
    """Calls of every operand of every entry point: (name, positional arguments, keywords, {position: format})."""
    T, I, O, R, N = 70, 64, 80, 16, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, device="cuda").normal_(generator=g).to(dtype)      # noqa: E731
    rows = torch.tensor([0, 30, 66], dtype=torch.int32, device="cuda"), torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    X, dZ, A, B, S = normal(T, I), normal(T, O), normal(N, R, I), normal(N, R, O), normal(T, R, dtype=torch.float32)
    e4 = {n: normal(T, n, dtype=torch.float8_e4m3fn) for n in (I, O)}
    e5 = normal(T, O, dtype=torch.float8_e5m2)
    codes, scales = sste.checkpoint_pack(X)
    return [
        ("adapter_fwd", [X, *rows, A, B], {}, {0: sste.BF16, 3: sste.BF16, 4: sste.BF16}),
        ("adapter_fwd", [e4[I], *rows, A, B], dict(dtype=sste.F8E4M3), {0: sste.F8E4M3}),
        ("adapter_dgrad", [dZ, *rows, A, B], {}, {0: sste.BF16, 3: sste.BF16, 4: sste.BF16}),
        ("adapter_dgrad", [e4[O], *rows, A, B], dict(dtype=sste.F8E4M3), {0: sste.F8E4M3}),
        ("adapter_dgrad", [e5, *rows, A, B], dict(dtype=sste.F8E5M2), {0: sste.F8E5M2}),
        ("adapter_wgrad", [dZ, X, S, S, *rows, N], {}, {0: sste.BF16, 1: sste.BF16}),
        ("adapter_wgrad", [e5, e4[I], S, S, *rows, N], dict(dtype=sste.F8E5M2, x_dtype=sste.F8E4M3), {0: sste.F8E5M2, 1: sste.F8E4M3}),
        ("adapter_wgrad", [e4[O], codes, S, S, *rows, N], dict(dtype=sste.F8E4M3, x_dtype=sste.F8BLOCK, x_blocks=scales), {0: sste.F8E4M3, 1: sste.F8BLOCK}),
        ("checkpoint_pack", [X], {}, {0: sste.BF16}),
        ("checkpoint_backward", [codes, scales], {}, {0: sste.F8BLOCK}),
    ]


@pytest.mark.gpu
@pytest.mark.parametrize("native", [False, True])
@pytest.mark.parametrize("number", range(10))
def test_operands_of_every_call(native, number):
    name, args, kw, operands = arguments()[number]
    call = getattr(sste, name) if native else binding._PYTHON[name]
    want = call(*args, **kw)
    for position, kind in operands.items():
        given = args[position]
        for dtype in ALL:
            if dtype.itemsize != OWN[kind].itemsize:
                continue
            args[position] = given.view(dtype)
            if dtype == OWN[kind] or dtype in RAW[dtype.itemsize]:
                assert all(a is b or torch.equal(a, b) for a, b in zip(call(*args, **kw), want)), (position, dtype)
            else:
                with pytest.raises(ValueError, match="must be .* not " + str(dtype)):
                    call(*args, **kw)
        args[position] = given
