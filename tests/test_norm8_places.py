"""Results in the place of an operand of another type (or of another result): refused before anything is launched (no GPU needed).

A row of such a result lies over other rows of the operand, which other blocks may still have to read."""
import ctypes

import pytest

from paper_2504_03871_amd import binding as B

S = ctypes.c_void_p(0)
X, R, H, Y, G, RS, DY, ADD, DH, DX = (0x10000 * i for i in range(1, 11))   # aligned addresses that are never dereferenced
HALF = [B.DTYPE_BF16, B.DTYPE_F16]


def overlaps(fn, *a, **kw):
    with pytest.raises(B.MoeError) as ei:
        fn(*a, **kw)
    assert ei.value.code == -8, ei.value


@pytest.mark.parametrize("T, d", [(1, 8), (2, 64), (5000, 4096)])
@pytest.mark.parametrize("dtype", HALF)
def test_forward(dtype, T, d):
    norm = B.make_norm(T, d, dtype, B.DTYPE_F32)

    def call(x=X, r=R, h=H, y=Y):
        B.moe_norm_fwd(norm, None, x, r, G, h, RS, y, None, None, stream=S)
    overlaps(call, h=X)
    overlaps(call, y=R)
    overlaps(call, y=R, h=None)
    overlaps(call, y=H)


@pytest.mark.parametrize("T, d", [(1, 8), (2, 64), (5000, 4096)])
@pytest.mark.parametrize("dtype", HALF)
def test_backward(dtype, T, d):
    norm = B.make_norm(T, d, dtype, B.DTYPE_F32)

    def call(dy=DY, h=H, add=ADD, dh=DH, dx=DX):
        B.moe_norm_bwd(norm, None, dy, h, G, RS, add, dh, dx, None, 0, None, stream=S)
    overlaps(call, dx=H)
    overlaps(call, dx=H, dh=None)
    overlaps(call, dh=DY)
    overlaps(call, dh=DY, dx=None)
    overlaps(call, dx=ADD)


def test_codes_have_a_place_of_their_own():
    norm = B.make_norm(5, 64)
    for at in (X, R, H, Y):
        overlaps(B.moe_norm_fwd, norm, None, X, R, G, H, RS, Y, at, RS, stream=S)
    overlaps(B.moe_quant_rows, B.DTYPE_BF16, 5, 64, 64, X, X, RS, stream=S)


def test_drop_s_step_is_a_whole_number():
    """64 bits of another kind would name a mask by their pattern."""
    import torch

    class OnGpu(torch.Tensor):
        is_cuda = True
    made = lambda dtype: torch.zeros(2, dtype=dtype).as_subclass(OnGpu)  # noqa: E731
    assert B.make_drop(0.1, 1, 0, made(torch.int64)).step
    for dtype in (torch.float64, torch.complex64, torch.int32, torch.float32):
        with pytest.raises(ValueError):
            B.make_drop(0.1, 1, 0, made(dtype))
