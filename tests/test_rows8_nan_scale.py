"""A scale byte of 255 stands for NaN, in what the rows show and in products of both result types."""
import pytest
import torch

from paper_2608_11235_amd import Rows8, quantize_rows, rows8_product
from tests.gpu_common import log_case, require_gpu


def place(r, block, cols):
    """of the scale of a row's block (the documented layout)"""
    return (r // 16 * -(-cols // 512) + block // 4) * 64 + r % 16 * 4 + block % 4


def test_values():
    x = Rows8(20, 700, device="cpu")
    x.data.fill_(0x38)  # 1.0
    x.scale[place(17, 5, 700)] = 255
    x.scale[place(3, 0, 700)] = 254
    v = x.values()
    bad = torch.zeros_like(v, dtype=torch.bool)
    bad[17, 640:] = True
    assert torch.equal(v.isnan(), bad)
    assert (v[3, :128] == 2.0 ** 127).all() and (v[4] == 1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(3, 40, 300), (30, 500, 700), (64, 200, 700), (200, 150, 700), (300, 257, 513), (40, 70, 8192)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products(M, N, K, dtype):
    """Rows with such a scale are NaN throughout, blocks of zeros with it too; the others keep their numbers."""
    require_gpu()
    log_case(f"scales of 255: {M} x {N} x {K} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(K)
    x, y = torch.randn((M, K), generator=g, device="cuda"), torch.randn((N, K), generator=g, device="cuda")
    x[2, :128] = 0
    a, w = quantize_rows(x), quantize_rows(y)
    alone = rows8_product(a, w, dtype=dtype)
    last = (K - 1) // 128
    a.scale[place(2, 0, K)] = 255
    w.scale[place(N - 1, last, K)] = 255
    w.scale[place(17, 1, K)] = 255
    got = rows8_product(a, w, dtype=dtype)
    rows, cols = torch.arange(M, device="cuda") != 2, torch.ones(N, dtype=torch.bool, device="cuda")
    cols[17] = cols[N - 1] = False
    assert got[2].isnan().all() and got[:, 17].isnan().all() and got[:, N - 1].isnan().all()
    assert torch.equal(got[rows][:, cols], alone[rows][:, cols])
