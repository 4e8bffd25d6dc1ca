"""8-bit rows against their definition, bit for bit, and their products against 64 bits."""
import math

import pytest
import torch

from paper_2608_11235_amd import Rows8, quantize_rows, rows8_product, rows8_product_workspace
from tests.gpu_common import log_case, require_gpu
from tests.rows8_ref import held, product, quantized

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def no_nan(x):
    return torch.nan_to_num(x, nan=0.0, posinf=math.inf, neginf=-math.inf)


def check_quantized(x):
    q = quantize_rows(x)
    v, e = held(q)
    want, we = quantized(x)
    R, K = x.shape
    assert torch.equal(e[:R, :we.shape[1]], we)
    assert (e[R:] == 0).all() and (e[:, we.shape[1]:] == 0).all()
    got = v[:R, :want.shape[1]]
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(no_nan(got), no_nan(want))
    assert (v[R:] == 0).all()
    assert torch.equal(q.values().isnan(), want[:, :K].isnan())
    # (fp32's largest numbers round up to 2^128, which it holds as infinity)
    full = no_nan(want[:, :K]) * torch.exp2(we.double()).repeat_interleave(128, 1)[:, :K]
    assert torch.equal(no_nan(q.values()), full.float())
    return q


@pytest.mark.parametrize("R,K", [(1, 1), (1, 127), (3, 128), (16, 129), (17, 512), (33, 513), (5, 1000), (300, 64),
                                 (64, 2047), (2, 18944), (1031, 640)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantized_rows(R, K, dtype):
    require_gpu()
    log_case(f"quantize {R} x {K} {dtype}")
    g = gen(R * 31 + K)
    x = torch.randn((R, K), generator=g, device="cuda") * torch.exp(3 * torch.randn((R, 1), generator=g, device="cuda"))
    x[:, ::7] *= 50
    check_quantized(x.to(dtype))


@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 8), (5, 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_and_unaligned_rows(offset, pad, dtype):
    require_gpu()
    big = torch.randn((37, offset + 300 + pad), generator=gen(offset), device="cuda").to(dtype)
    log_case(f"quantize strided offset {offset} pad {pad} {dtype}")
    check_quantized(big[:, offset:offset + 300])
    check_quantized(big[::2, offset:offset + 300])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_of_every_kind(dtype):
    """Zeros, subnormal and huge numbers, halves of a step, 448 and the next above it, NaN and infinities."""
    require_gpu()
    log_case(f"quantize special values {dtype}")
    tiny = torch.finfo(dtype).tiny
    x = torch.randn((40, 384), generator=gen(9), device="cuda").double()
    x[0] = 0
    x[1, :128] = 0
    x[2] *= tiny
    x[3] = 1e-45 if dtype is torch.float32 else 2.0 ** -133
    x[4] *= torch.finfo(dtype).max / 8
    x[5, 7] = torch.finfo(dtype).max
    x[6, 0], x[6, 130], x[6, 260] = 448, 450, 2.0 ** 8 * 1.75 * 2.0 ** -20
    x[7, 3], x[8, 200], x[9, 300] = math.nan, math.inf, -math.inf
    x[10, :128] = math.inf
    x[11] = torch.arange(384, device="cuda") / 16.0    # every half of a step of small numbers
    x[12, 0] = 448
    x[12, 1:128] = torch.arange(1, 128, device="cuda") * 2.0 ** -11   # subnormal results, ties among them
    x[13] = -0.0
    x[14] *= torch.exp2(torch.randint(-126, 120, (384,), generator=gen(2), device="cuda").double())
    check_quantized(x.to(dtype))


def test_every_bf16_number():
    """All 65536 patterns, each beside 448 and beside 1."""
    require_gpu()
    log_case("quantize every bf16")
    x = torch.arange(-32768, 32768, device="cuda").short().view(torch.bfloat16).view(-1, 64)
    for c in (448.0, 1.0):
        check_quantized(torch.cat([x, torch.full((1024, 64), c, device="cuda", dtype=torch.bfloat16)], 1))


def check_product(a, w, bias=None, dtype=torch.bfloat16, out=None):
    got = rows8_product(a, w, bias=bias, dtype=dtype, out=out)
    want, sums, eight = product(a, w, bias)
    ok = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    d = (got.double() - want)[ok].abs()
    if got.dtype is torch.float32:
        tol = sums + 2.0 ** -24 * want.abs() + 2.0 ** -148
    else:
        tol = sums + eight + 2.0 ** -8 * want.abs() + 2.0 ** -133
    assert (d <= tol[ok]).all(), float((d - tol[ok]).max())
    return got, want


def rows(seed, R, K, spread=0.5):
    g = gen(seed)
    x = torch.randn((R, K), generator=g, device="cuda") * torch.exp(spread * torch.randn((R, K), generator=g, device="cuda"))
    return quantize_rows(x)


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 5, 64), (2, 17, 129), (15, 100, 512), (16, 688, 256), (17, 257, 513),
          (31, 1, 1000), (32, 500, 4096), (33, 48, 640), (48, 63, 2048), (64, 1000, 1536), (65, 130, 127),
          (130, 65, 1024), (333, 1531, 1000), (257, 1, 300), (128, 128, 8192), (700, 520, 640), (4, 9000, 64),
          (1024, 512, 1024), (2047, 300, 4097), (2533, 6750, 895), (2533, 6751, 895), (2346, 3703, 603)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products(M, N, K, dtype):
    require_gpu()
    log_case(f"product {M} x {N} x {K} {dtype}")
    bias = torch.randn(N, generator=gen(3), device="cuda") if (M + N) % 2 else None
    got, want = check_product(rows(M, M, K), rows(N + 1, N, K), bias, dtype)
    # half a step of bf16 is 2^-8 of a value at the most
    assert (got.double() - want).norm() <= (2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -20) * want.norm()


@pytest.mark.parametrize("M", [3, 40, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_row_that_is_not_finite_stays_alone(M, dtype):
    require_gpu()
    log_case(f"NaN rows, {M} {dtype}")
    x = torch.randn((M, 700), generator=gen(1), device="cuda")
    y = torch.randn((200, 700), generator=gen(2), device="cuda")
    x[1, 650], y[17, 3] = math.inf, math.nan
    got, _ = check_product(quantize_rows(x), quantize_rows(y), dtype=dtype)
    bad = torch.isnan(got)
    assert bad[1].all() and bad[:, 17].all() and int(bad.sum()) == 200 + M - 1


@pytest.mark.parametrize("M", [5, 64, 200])
@pytest.mark.parametrize("up,down", [(100, -110), (-60, 70), (40, 55)])
def test_scales_far_apart(M, up, down):
    """Blocks whose scales are many powers of two apart, and products near the ends of fp32."""
    require_gpu()
    log_case(f"scales 2^{up}, 2^{down}, {M} rows")
    x = torch.randn((M, 512), generator=gen(4), device="cuda") * 2.0 ** up
    y = torch.randn((96, 512), generator=gen(5), device="cuda") * 2.0 ** down
    x[:, 128:256] *= 2.0 ** -30 if up > 0 else 2.0 ** 30
    y[::2, 128:256] *= 2.0 ** 20
    for dtype in (torch.bfloat16, torch.float32):
        check_product(quantize_rows(x), quantize_rows(y), dtype=dtype)


@pytest.mark.parametrize("M,N,K", [(20, 40, 900), (300, 257, 513), (333, 500, 4096), (1000, 900, 700)])
@pytest.mark.parametrize("up,down", [(0, 0), (90, 0), (-90, 0), (90, -110), (-90, -50), (50, 51), (-51, 60)])
def test_far_scales_in_a_few_rows(M, N, K, up, down):
    """Rows of numbers far from one, some of whose products fall below the normal numbers, beside ordinary ones."""
    require_gpu()
    log_case(f"far rows 2^{up}, 2^{down}: {M} x {N} x {K}")
    x, y = torch.randn((M, K), generator=gen(6), device="cuda"), torch.randn((N, K), generator=gen(7), device="cuda")
    x[M // 2] *= 2.0 ** up
    x[M // 3, :K // 2] *= 2.0 ** up
    y[N // 2] *= 2.0 ** down
    y[N - 1, K // 3:] *= 2.0 ** down
    for dtype in (torch.bfloat16, torch.float32):
        check_product(quantize_rows(x), quantize_rows(y), dtype=dtype)


@pytest.mark.parametrize("M,N,K", [(7, 33, 300), (70, 130, 1000), (300, 257, 513)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 1), (4, 4), (3, 2)])
def test_strided_output_keeps_what_lies_between(M, N, K, dtype, pad, offset):
    require_gpu()
    log_case(f"strided out {M} x {N} {dtype} pad {pad} offset {offset}")
    a, w = rows(1, M, K), rows(2, N, K)
    big = torch.full((M + 2, offset + N + pad), 7.0, dtype=dtype, device="cuda")
    out = big[1:M + 1, offset:offset + N]
    check_product(a, w, dtype=dtype, out=out)
    big[1:M + 1, offset:offset + N] = 7.0
    assert (big == 7.0).all()


def test_no_rows():
    require_gpu()
    a, w = Rows8(0, 128), rows(1, 5, 128)
    assert rows8_product(a, w).shape == (0, 5) and rows8_product(w, a).shape == (5, 0)
    assert quantize_rows(torch.zeros((0, 7), device="cuda")).rows == 0


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (32, 688, 2048), (300, 256, 4096)])
def test_graph_streams_and_workspace(M, N, K):
    """Captured and replayed between eager work, on a stream of its own, with a workspace of the caller's."""
    require_gpu()
    log_case(f"graph {M} x {N} x {K}")
    x = torch.randn((M, K), generator=gen(1), device="cuda").to(torch.bfloat16)
    w = rows(2, N, K)
    a = quantize_rows(x)
    n = rows8_product_workspace(a, w)
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    rows8_product(a, w, out=out, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        quantize_rows(x, out=a)
        rows8_product(a, w, out=out, workspace=ws)
    s = torch.cuda.Stream()
    for rep in range(4):
        x.copy_(torch.randn((M, K), generator=gen(10 + rep), device="cuda"))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            s.wait_stream(torch.cuda.default_stream())
            eager = rows8_product(quantize_rows(x), w)
        other = rows8_product(quantize_rows(x, stream=s), w, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(out, other), rep


def test_rows_do_not_depend_on_the_others():
    require_gpu()
    for M in (20, 150):
        x = torch.randn((M, 1024), generator=gen(1), device="cuda")
        w = rows(2, 500, 1024)
        one = rows8_product(quantize_rows(x), w)
        x[3:] = torch.randn((M - 3, 1024), generator=gen(7), device="cuda") * 100
        assert torch.equal(rows8_product(quantize_rows(x), w)[:3], one[:3])


def test_refusals():
    require_gpu()
    from paper_2608_11235_amd._lib import CoraError
    a, w = rows(1, 4, 256), rows(2, 6, 256)
    with pytest.raises(ValueError, match="columns"):
        rows8_product(a, rows(3, 6, 128))
    with pytest.raises(TypeError, match="dtype"):
        rows8_product(a, w, dtype=torch.float16)
    with pytest.raises(ValueError, match="out"):
        rows8_product(a, w, out=torch.empty((4, 7), device="cuda"))
    with pytest.raises(TypeError, match="bias"):
        rows8_product(a, w, bias=torch.zeros(6, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="bias"):
        rows8_product(a, w, bias=torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError, match="out"):
        quantize_rows(torch.zeros((4, 128), device="cuda"), out=a)
    with pytest.raises(ValueError, match="column"):
        quantize_rows(torch.zeros((4, 0), device="cuda"))
    with pytest.raises(ValueError, match="strides"):
        quantize_rows(torch.zeros((4, 256), device="cuda")[:, ::2])
    with pytest.raises(CoraError) as e:
        Rows8(4, (1 << 20) + 1)
    assert e.value.status == -2
    n = rows8_product_workspace(a, w)
    if n:
        with pytest.raises(CoraError):
            rows8_product(a, w, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
