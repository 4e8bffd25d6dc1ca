"""8-bit products of sizes that reach every way a product is made: columns over several workgroups and their sums, each kind
of registers' share for few rows, every tile, a second launch of other tiles.  test_rows8_plan.py says which they reach."""
import numpy as np
import pytest
import torch

import seeded_inputs as si
from paper_2608_11235_amd import Chunk, Model, cache_plan, quantize_rows, rows8_product
from tests.gpu_common import log_case, require_gpu
from tests.rows8_ref import product
from tests.test_gpu_cached_pass import cache_for, masked_logits, put
from tests.test_gpu_quantized_pass import quantized_logits, values

pytestmark = pytest.mark.gpu

SHAPES = [(1, 700, 12288), (16, 130, 5000), (5, 257, 18944), (13, 8301, 512), (17, 40, 4500), (32, 515, 12288),
          (30, 301, 18944), (32, 8937, 512), (64, 130, 12288), (48, 67, 18944), (1, 1, 8401), (33, 1, 4431), (9, 50, 600), (20, 70, 640), (70, 100, 700),
          (143, 54305, 318), (136, 70644, 943), (73, 77398, 1447), (92, 71556, 978), (791, 41340, 2436), (2336, 14852, 2621),
          (1459, 5639, 1861), (5067, 3562, 2908), (267, 16024, 16258), (268, 8015, 15555), (6556, 546, 422), (5487, 283, 4355),
          (5605, 130, 6962), (4112, 1, 10027), (74, 36719, 538), (86, 17279, 3982), (67, 8485, 5630), (66, 4336, 7920),
          (66, 16834, 1), (290, 10754, 11718), (520, 3158, 19403), (2594, 258, 14151), (65, 8932, 1), (129, 8915, 22924),
          (2067, 68, 4579), (1047, 67, 8657), (4590, 1, 3800), (78, 1, 2377), (84, 1, 4124), (40, 3, 1935), (46, 1, 1836)]


def rows(seed, R, K):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((R, K), generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn((R, K), generator=g, device="cuda"))
    return quantize_rows(x)


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products(M, N, K, dtype):
    """Within what 32-bit sums, the 8-bit instruction (bf16 results) and one rounding may be off by; again with the same bits,
    and into rows of another stride."""
    require_gpu()
    log_case(f"product {M} x {N} x {K} {dtype}")
    a, w = rows(M, M, K), rows(N + 1, N, K)
    bias = torch.randn(N, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") if (M + N) % 2 else None
    got = rows8_product(a, w, bias=bias, dtype=dtype)
    big = torch.full((M, N + 3), 7.0, dtype=dtype, device="cuda")
    rows8_product(a, w, bias=bias, out=big[:, 1:N + 1])
    assert torch.equal(big[:, 1:N + 1], got) and (big[:, 0] == 7).all() and (big[:, N + 1:] == 7).all()
    want, sums, eight = product(a, w, bias)
    off = sums + 2.0 ** -24 * want.abs() if dtype is torch.float32 else sums + eight + 2.0 ** -8 * want.abs()
    assert ((got.double() - want).abs() <= off).all()
    # what the roundings amount to: half a step of the result's type
    assert (got.double() - want).norm() <= (2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -20) * want.norm()


# (width, heads, kv heads, inner width, rows)
LAYERS = [(256, 8, 2, 12288, 1), (256, 8, 2, 18944, 16), (256, 8, 2, 12288, 30), (256, 8, 2, 18944, 32), (256, 8, 2, 12288, 64),
          (320, 8, 2, 18944, 48), (256, 8, 2, 12288, 70), (256, 8, 2, 4224, 100), (4160, 8, 2, 64, 64), (4160, 8, 2, 300, 33),
          (4160, 8, 2, 64, 100), (8192, 8, 2, 64, 100), (256, 40, 8, 256, 64), (256, 40, 8, 256, 100), (512, 36, 4, 512, 90),
          (7168, 8, 2, 128, 64), (7168, 8, 2, 128, 20)]


@pytest.mark.parametrize("d,heads,kv,ffn,rows", LAYERS)
def test_one_layer(d, heads, kv, ffn, rows):
    """Requests of one key, whose attention's output is v itself: what differs from the definition in 64 bits is that fp32 sums,
    off by 5e-5 at the most, move a bf16 number in 1 % of the cases and the 8-bit number behind it in 3 % of these; one of
    1000 numbers that moves by a step is a tenth of what 8 bits change in a product.  The logits' own rounding is 2^-9 of
    them, 0.03 of the 0.07 that 8 bits change.  Half the rows stay below 0.15."""
    require_gpu()
    log_case(f"quantized layer d={d} heads={heads} ffn={ffn} rows={rows}")
    spec = si.ModelSpec("one", 1, d, heads, kv, 128, ffn, 900, 5, bool(ffn % 256), 1e-6, 1e6, 4.0)
    cache, chunk = cache_for(spec, rows, 8), Chunk(rows, rows)
    put(chunk.count, [1] * rows)
    cache_plan(cache, chunk)
    tokens = np.random.default_rng(rows).integers(0, spec.vocab, size=rows)
    tok = torch.as_tensor(tokens.astype(np.int32)).cuda()
    with Model(spec, 0, 4, 128) as m:
        w8 = m.quantize()
        got = values(m.forward_cached(cache, chunk, tok, causal=True, weights=w8))
        again = values(m.forward_cached(cache, chunk, tok, causal=True, weights=w8))
    assert np.array_equal(got, again)
    pick = np.unique(np.linspace(0, rows - 1, min(rows, 15)).astype(int))
    w, alone = si.HostWeights(spec, 0), np.eye(len(pick), dtype=bool)
    want, full = quantized_logits(w, spec, tokens[pick], alone), masked_logits(w, spec, tokens[pick], alone)
    ratio = np.linalg.norm(got[pick] - want, axis=1) / np.linalg.norm(want - full, axis=1)
    log_case(f"  {np.round(sorted(ratio), 3)}")
    assert np.median(ratio) <= 0.15 and max(ratio) <= 0.75
