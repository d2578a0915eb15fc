"""Activations of the products in 8 bits over all the numbers of a type: off by the rounding of the result, also where they are next to zero."""
import numpy as np
import pytest
from scipy.special import log_ndtr

from paper_2504_03871_amd import binding as B
from tests.test_gpu_norm8 import ACT, DEV, TD, U, dev, empty, f64, half_step, least, linear8, near

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def numbers(dtype, lo, hi):
    """Every number of a 16-bit type from lo to hi, a grid of fp32's, filled up to a multiple of 64 (by the last)."""
    if dtype == "f32":
        v = np.linspace(lo, hi, 50000).astype(np.float32)
    else:
        v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TD[dtype]).double().numpy()
        v = np.sort(v[np.isfinite(v) & (v >= lo) & (v <= hi)])
    return np.concatenate([v, np.full(-v.size % 64, v[-1])]).astype(np.float64)


@pytest.mark.parametrize("T, K", [(1, 64), (20, 64), (40, 64), (40, 4096), (300, 64)])     # strips, pairs of them, tiles, K parts
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
def test_activation_of_every_number(act, dtype, T, K):
    """Codes of zero, so that z is the bias; the second of SwiGLU's two is one."""
    # down to where the results leave fp32's normal numbers (gelu: exp(-z^2 / 2), swiglu: the reciprocal of exp(-z))
    z = numbers(dtype, -12.5 if act == "gelu" else -80, 100)
    N, mats = z.size, 1 if act == "gelu" else 2
    x, w = torch.zeros(T, K, dtype=torch.int8, device=DEV), [torch.zeros(K * N, dtype=torch.int8, device=DEV) for _ in range(mats)]
    b = [dev(z, dtype)] + [torch.ones(N, dtype=TD[dtype], device=DEV)] * (mats - 1)
    y = linear8(T, K, N, dtype, act, x, torch.ones(T, device=DEV), w, [torch.ones(N, device=DEV)] * mats, b, None, empty(T, N, dtype=dtype))
    want = z * np.exp(log_ndtr(z)) if act == "gelu" else z / (1 + np.exp(-z))
    # The argument of an exponential, up to z^2 / 2 or |z|, comes from four roundings of fp32, and they are its relative error; all else are 20 more.
    # 16 bits, GELU: its approximation's 4e-6 besides.
    rel = (4 * (z * z / 2 if act == "gelu" else np.abs(z)) + 20) * U + (4e-6 if act == "gelu" and dtype != "f32" else 0)
    want = np.broadcast_to(want, (T, N))
    near(act, y, want, (rel + half_step(dtype) * (1 + rel)) * np.abs(want) + least(dtype))
    assert (f64(y) == f64(y)[:1]).all()
