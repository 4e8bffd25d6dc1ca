"""The paged cache's operators over their range of sizes: requests in several key ranges, one very
long request, thousands of short ones, and chunks large enough for a store's threads to take more
heads."""
import numpy as np
import pytest
import torch

from paper_2608_11235_amd import Chunk, KVCache, cache_attention, cache_plan, cache_store, rope_table
from tests import cache_ref as ref
from tests.gpu_common import log_case, require_gpu
from tests.test_gpu_cache import compare, filled, put, requests

pytestmark = pytest.mark.gpu

# lengths around the ends of ranges of 640 and 1280 keys, of the 1.25 ranges that stay whole, and of
# groups and tiles of keys inside them
LENS = [1, 639, 640, 641, 800, 801, 1280, 1281, 1600, 1601, 2561, 33, 5000, 9001]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,Hkv,count", [(7, 1, 1), (28, 4, 1), (28, 4, 4), (4, 4, 17), (8, 2, 16), (6, 3, 60)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("max_len", [0, 700])
def test_attention_key_ranges(hd, H, Hkv, count, causal, max_len):
    require_gpu()
    rng = np.random.default_rng(hd + H + count)
    log_case(f"ranges hd={hd} H={H}/{Hkv} count={count} causal={causal} max_len={max_len}")
    counts = np.minimum(LENS, count)
    compare(*requests(rng, LENS, counts, hd, H, Hkv, 64), causal, max_count=count, max_len=max_len)


@pytest.mark.parametrize("hd,H,Hkv", [(64, 4, 1), (128, 8, 2)])
@pytest.mark.parametrize("count", [1, 30])
@pytest.mark.parametrize("max_len", [0, 1000])
def test_attention_one_long_request(hd, H, Hkv, count, max_len):
    require_gpu()
    rng = np.random.default_rng(hd + count)
    log_case(f"long hd={hd} count={count} max_len={max_len}")
    compare(*requests(rng, [70001], [count], hd, H, Hkv, 128), True, max_count=count, max_len=max_len)


@pytest.mark.parametrize("B,max_count", [(1025, 3), (4096, 3), (4096, 40)])
def test_attention_thousands_of_requests(B, max_count):
    """The largest batch, and both kernels' way of finding a request."""
    require_gpu()
    rng = np.random.default_rng(B)
    lens = rng.integers(1, 6, size=B)
    lens[B // 2] = 1500
    count = np.minimum(lens, rng.integers(0, 4, size=B))
    log_case(f"requests B={B} max_count={max_count}")
    compare(*requests(rng, lens, count, 64, 2, 1, 32), True, max_count=max_count, max_len=1500)


def test_attention_requests_without_rows():
    """Nothing to do at all: the list of work is empty and out stays as it is."""
    require_gpu()
    rng = np.random.default_rng(1)
    cache, chunk, q, ks, vs, T = requests(rng, [300, 40], [0, 0], 128, 4, 2, 64, rows=5)
    for max_count in (1, 100):
        out = torch.full_like(q, 9.0)
        cache_attention(cache, 0, q, chunk, max_count=max_count, out=out)
        assert (out == 9).all()


@pytest.mark.parametrize("max_count,max_len", [(1, 1), (1, 9000), (30, 9000), (30, 300), (0, 0)])
def test_attention_rows_before_the_first_request(max_count, max_len):
    """cu need not start at 0: rows of no request stay as they are."""
    require_gpu()
    rng = np.random.default_rng(2)
    lens, count = [900, 2100, 64, 7], [40, 3, 64, 1]
    cache, chunk, q, ks, vs, T = requests(rng, lens, count, 64, 8, 2, 32, rows=sum(count) + 20)
    want = torch.full_like(q, 9.0)
    cache_attention(cache, 0, q, chunk, causal=True, out=want, max_count=max_count, max_len=max_len)
    for late in (1, 5, 20):
        shifted = torch.zeros_like(q)
        shifted[late:late + T] = q[:T]
        chunk.cu.add_(late)
        out = torch.full_like(q, 9.0)
        cache_attention(cache, 0, shifted, chunk, causal=True, out=out, max_count=max_count, max_len=max_len)
        chunk.cu.sub_(late)
        assert (out[:late] == 9).all() and (out[late + T:] == 9).all()
        assert torch.equal(out[late:late + T], want[:T])


def test_attention_expected_lengths_that_grow():
    """A max_len of its own for every call: the sizes kept on the host stay few, results the same."""
    require_gpu()
    rng = np.random.default_rng(4)
    cache, chunk, q, ks, vs, T = requests(rng, [300, 40], [1, 1], 64, 4, 2, 64)
    want = cache_attention(cache, 0, q, chunk, max_count=1, max_len=1)
    for n in range(2, 600):
        got = cache_attention(cache, 0, q, chunk, max_count=1, max_len=n)
    assert torch.equal(got, want) and len(cache._workspaces) <= 256


@pytest.mark.parametrize("page", [1 << 27, (1 << 27) + 1, -(1 << 27), 4, -1])
@pytest.mark.parametrize("rows", [8, 9000])
def test_plan_pages_that_are_not_there(page, rows):
    """A page number whose slots would wrap around to those of another request gives no slot."""
    require_gpu()
    cache, chunk = KVCache(1, 4, 1, 64, 32, 1, 3), Chunk(1, rows)
    put(cache.table, [[page, 1, 2]]); put(cache.len, [40])
    put(chunk.start, [30]); put(chunk.count, [4])
    cache_plan(cache, chunk)
    assert chunk.status.tolist() == [0] and chunk.positions[:5].tolist() == [30, 31, 32, 33, -1]
    assert chunk.slots[:5].tolist() == [-1, -1, 32, 33, -1]
    cache.k.zero_(); cache.v.zero_()
    x = torch.ones((rows, 3 * 64), dtype=torch.bfloat16, device="cuda")
    q = cache_store(cache, 0, x, 1, chunk)
    used = ref.natural(cache.k[0], ref.offsets(32, 64)[0])
    assert (q[:2] == 0).all() and (used[1, 0, :2] == 1).all() and int((used != 0).sum()) == 2 * 64


@pytest.mark.parametrize("H,Hkv", [(9, 3), (13, 13)])
@pytest.mark.parametrize("f32", [False, True])
def test_store_large(H, Hkv, f32):
    """More than 4096 windows x heads; heads that four do not divide; runs that straddle windows."""
    require_gpu()
    hd, page, rows, B = 128, 64, 11050, 3
    assert -(-rows // 32) * (H + Hkv) >= 4096
    log_case(f"store large H={H}/{Hkv} f32={f32}")
    rng = np.random.default_rng(H)
    cache = filled(1, 190, Hkv, hd, page, B, 80, rng)
    chunk = Chunk(B, rows)
    first, count = np.array([5, 0, 3]), np.array([4000, 3001, 4003])
    put(chunk.count, first)
    cache_plan(cache, chunk, reset=True)
    put(chunk.start, first); put(chunk.count, count)
    cache_plan(cache, chunk)
    T = int(count.sum())
    gen = torch.Generator(device="cuda").manual_seed(H)
    x = torch.randn((rows, (H + 2 * Hkv) * hd), generator=gen, device="cuda")
    x = x if f32 else x.to(torch.bfloat16)
    rope = rope_table(4100, hd, 1e4)
    v0 = cache.v.clone()
    q = torch.full((rows, H, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    cache_store(cache, 0, x, H, chunk, rope=rope, q=q)
    pos, slots = chunk.positions[:T].long(), chunk.slots[:T].long()
    assert len(set(slots.tolist())) == T
    xx = x[:T].double().reshape(T, H + 2 * Hkv, hd)
    a, b = xx[:, :H + Hkv, :hd // 2], xx[:, :H + Hkv, hd // 2:]
    c, s = (rope.double()[pos][:, None, :, i] for i in range(2))
    want = torch.cat([a * c - b * s, b * c + a * s], -1)
    # two products and a sum in fp32 (2^-24 each of the magnitudes), one rounding to bf16 (2^-8)
    mag = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)
    tol = 2.0 ** -8 * want.abs() + 3 * 2.0 ** -24 * mag * (1 + 2.0 ** -8)
    assert ((q[:T].double() - want[:, :H]).abs() <= tol[:, :H]).all()
    assert (q[T:] == 7).all()
    ko, vo = ref.offsets(page, hd)
    kn, vn, vn0 = ref.natural(cache.k[0], ko), ref.natural(cache.v[0], vo), ref.natural(v0[0], vo)
    got_k = kn[slots // page, :, slots % page].double()
    assert ((got_k - want[:, H:]).abs() <= tol[:, H:]).all()
    assert torch.equal(vn[slots // page, :, slots % page], xx[:, H + Hkv:].to(torch.bfloat16))
    vn[slots // page, :, slots % page] = 0
    vn0[slots // page, :, slots % page] = 0
    assert torch.equal(vn, vn0)
