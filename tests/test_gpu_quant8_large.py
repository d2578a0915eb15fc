"""Weights to 8 bits at the sizes of real layers: many blocks of columns, and more than 2^31 bytes over the experts."""
import pytest

from paper_2504_03871_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.mark.parametrize("n, K, N", [(1, 14336, 4096), (2, 64, 65536), (2, 65536, 64), (5, 16384, 32768)])
def test_quantised_weights_by_torch_s_own_arithmetic(n, K, N):
    g = torch.Generator(device=DEV)
    g.manual_seed(n + K + N)
    W = torch.empty(n, K, N, dtype=torch.bfloat16, device=DEV)
    for w in W:
        w.copy_(torch.randn(K, N, generator=g, device=DEV))
    codes, scales = torch.full((n * K * N + 64,), 99, dtype=torch.int8, device=DEV), torch.empty(n, N, device=DEV)
    B.moe_quant_weight(B.DTYPE_BF16, n, K, N, W, codes, scales)
    assert bool((codes[n * K * N:] == 99).all())
    for i in {0, n // 2, n - 1}:
        top = W[i].abs().amax(dim=0).float()
        assert torch.equal(scales[i], top * torch.tensor(1 / 127, dtype=torch.float32, device=DEV))
        up = torch.full_like(top, 127) / top      # (127 / top is torch's reciprocal, times 127: two roundings)
        laid = codes[i * K * N:(i + 1) * K * N].view(N // 16, K // 64, 4, 16, 16)     # column / 16, row / 64, row % 64 / 16, column % 16, row % 16
        for c in range(0, N, 4096):
            cols = slice(c, min(c + 4096, N))
            want = torch.round(W[i][:, cols].float() * up[cols]).to(torch.int8).view(K // 64, 4, 16, -1, 16).permute(3, 0, 1, 4, 2)
            wrong = int((laid[c // 16:c // 16 + want.shape[0]] != want).sum())
            assert wrong == 0, (i, c, wrong)
