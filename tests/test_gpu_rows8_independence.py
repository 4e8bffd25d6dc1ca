"""A product's results do not change with what the other rows of either operand hold, in both result types."""
import pytest
import torch

from paper_2608_11235_amd import quantize_rows, rows8_product
from tests.gpu_common import log_case, require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(20, 300, 1024), (40, 70, 1024), (64, 500, 700), (150, 500, 1024), (300, 257, 513), (48, 63, 8192),
                                   (2533, 6750, 895)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("power", [90, -90, 7])
def test_other_rows_far_from_one(M, N, K, dtype, power):
    """One row beside ordinary ones: the whole of it, or one block of columns, far from one."""
    require_gpu()
    log_case(f"far row beside others {M} x {N} x {K} {dtype} 2^{power}")
    g = torch.Generator(device="cuda").manual_seed(M + K)
    x, y = torch.randn((M, K), generator=g, device="cuda"), torch.randn((N, K), generator=g, device="cuda")
    a, w = quantize_rows(x), quantize_rows(y)
    alone = rows8_product(a, w, dtype=dtype)
    for row, cols in ((5, slice(None)), (M - 1, slice(K - 100, None)), (M // 2, slice(0, 128))):
        far = x.clone()
        far[row, cols] *= 2.0 ** power
        keep = torch.arange(M, device="cuda") != row
        assert torch.equal(rows8_product(quantize_rows(far), w, dtype=dtype)[keep], alone[keep]), row
    for row, cols in ((6, slice(None)), (N - 1, slice(0, 100)), (N // 2, slice(K - 128, None))):
        far = y.clone()
        far[row, cols] *= 2.0 ** power
        keep = torch.arange(N, device="cuda") != row
        assert torch.equal(rows8_product(a, quantize_rows(far), dtype=dtype)[:, keep], alone[:, keep]), row
