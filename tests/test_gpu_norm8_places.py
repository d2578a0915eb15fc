"""The norm's gradients in the place of h, of its own type, on the GPU: the bits of a call with places of its own."""
import pytest

from paper_2504_03871_amd import binding as B
from tests.test_gpu_norm8 import DEV, DT, U, empty, norm_case, norm_tolerance

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("T, d", [(3, 64), (700, 1091), (2048, 520), (3000, 256), (600, 8200)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_dx_over_h(T, d, dtype, p):
    x, h, g, dy, add = norm_case(T, d, dtype, dtype, 6)
    norm, drop = B.make_norm(T, d, DT[dtype]), B.make_drop(p, 3) if p else None
    rstd, y = empty(T), empty(T, d, dtype=dtype)
    B.moe_norm_fwd(norm, None, h, None, g, None, rstd, y, None, None)
    dh, dx, dg, ws = empty(T, d, dtype=dtype), empty(T, d, dtype=dtype), empty(d), torch.empty(B.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device=DEV)
    B.moe_norm_bwd(norm, drop, dy, h, g, rstd, add, dh, dx, dg, 0, ws)
    h2, dh2, dg2 = h.clone(), empty(T, d, dtype=dtype), empty(d)
    B.moe_norm_bwd(norm, drop, dy, h2, g, rstd, add, dh2, h2, dg2, 0, ws)
    assert torch.equal(dh2, dh) and torch.equal(h2, dx)
    # gamma's gradient may be added up in another order
    sums = (norm_tolerance(d) + (T + 40) * U) * (dy.double().abs() * (h.double() * rstd.double()[:, None]).abs()).sum(dim=0) + 1e-30
    assert bool(((dg2.double() - dg.double()).abs() <= 2 * sums).all())
