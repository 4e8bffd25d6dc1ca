"""The paged cache's operators against plain references: plans and slots equal, stores within the
rounding of their formula, attention within the rounding of its bf16 terms."""
import math

import numpy as np
import pytest
import torch

from paper_2608_11235_amd import (Chunk, KVCache, cache_attention, cache_attention_workspace,
                                  cache_plan, cache_store, rope_table)
from paper_2608_11235_amd._lib import CoraError
from tests import cache_ref as ref
from tests.gpu_common import log_case, require_gpu

pytestmark = pytest.mark.gpu


def put(t, a):
    t.copy_(torch.as_tensor(np.asarray(a)).to(t.dtype))


# ---- plan --------------------------------------------------------------------------------------
def same_plan(cache, chunk, host, out):
    for name in ("cu", "positions", "slots", "status"):
        assert getattr(chunk, name).cpu().numpy().tolist() == list(np.asarray(out[name])), name
    assert cache.len.cpu().numpy().tolist() == host.len.tolist()
    assert int(cache.n_free.cpu()) == len(host.free)
    assert cache.free.cpu().numpy().tolist()[:len(host.free)] == host.free
    table = cache.table.cpu().numpy()
    for b in range(host.B):
        n = -(-int(host.len[b]) // host.page)
        assert table[b, :n].tolist() == host.table[b, :n].tolist()


@pytest.mark.parametrize("B,page,max_pages,n_pages,rows", [
    (1, 32, 4, 4, 128), (3, 64, 5, 9, 100), (64, 32, 8, 200, 900), (70, 128, 3, 90, 20000),
    (1024, 32, 6, 3000, 9000), (1500, 256, 4, 2500, 60000), (4096, 64, 2, 3000, 8192)])
def test_plan_over_a_servers_life(B, page, max_pages, n_pages, rows):
    """Random arrivals, chunks, repeats, refusals and departures, every array compared each time."""
    require_gpu()
    log_case(f"plan B={B} page={page}")
    rng = np.random.default_rng(B)
    cache = KVCache(1, n_pages, 1, 64, page, B, max_pages)
    chunk, host = Chunk(B, rows), ref.Plan(B, max_pages, n_pages, page)
    for step in range(8):
        start, count = np.zeros(B, np.int64), np.zeros(B, np.int64)
        for b in range(B):
            kind = rng.integers(0, 12)
            n = int(host.len[b])
            if kind == 0:
                count[b] = -1
            elif kind == 1:
                start[b], count[b] = n + 1, 3          # a gap
            elif kind == 2:
                start[b], count[b] = -1, 2
            elif kind == 3:
                start[b], count[b] = n, max_pages * page - n + 1  # one past the table
            elif kind == 4:
                start[b], count[b] = rng.integers(0, n + 1), max(1, n // 2)
            elif kind >= 6:
                start[b] = n
                count[b] = rng.integers(1, max(2, rows // B * 2))
        put(chunk.start, start)
        put(chunk.count, count)
        reset = step == 5
        cache_plan(cache, chunk, reset=reset)
        same_plan(cache, chunk, host, host.step(start, count, rows, reset))


def test_plan_in_a_graph_with_changing_lengths():
    require_gpu()
    B, page, rows = 5, 32, 64
    cache, chunk = KVCache(1, 12, 1, 64, page, B, 6), Chunk(B, rows)
    host = ref.Plan(B, 6, 12, page)
    put(chunk.count, [1] * B)
    cache_plan(cache, chunk, reset=True)
    host.step([0] * B, [1] * B, rows, True)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        cache_plan(cache, chunk)
    rng = np.random.default_rng(1)
    for _ in range(6):
        start, count = host.len.copy(), rng.integers(-1, 30, size=B)
        put(chunk.start, start)
        put(chunk.count, count)
        g.replay()
        torch.cuda.synchronize()
        same_plan(cache, chunk, host, host.step(start, count, rows))


def test_plan_with_a_table_that_holds_nonsense():
    """Pages outside the pool are handed on, never followed: the rows' slots lie outside the cache
    and the store leaves them out."""
    require_gpu()
    cache, chunk = KVCache(1, 4, 1, 64, 32, 2, 2), Chunk(2, 8)
    cache.k.zero_(); cache.v.zero_()
    put(cache.table, [[-5, 9], [1000, 3]])
    put(cache.len, [20, 20])
    put(cache.n_free, [99])                           # more than there are: taken as 4
    put(cache.free, [7, -1, 2, 3])
    put(chunk.start, [18, 18]); put(chunk.count, [2, 2])
    cache_plan(cache, chunk)
    x = torch.ones((8, 3 * 64), dtype=torch.bfloat16, device="cuda")
    q = cache_store(cache, 0, x, 1, chunk)
    torch.cuda.synchronize()
    assert (cache.k == 0).all() and (cache.v == 0).all()
    assert (q[:4] == 0).all()


# ---- store -------------------------------------------------------------------------------------
def filled(n_layers, n_pages, Hkv, hd, page, B, max_pages, rng):
    cache = KVCache(n_layers, n_pages, Hkv, hd, page, B, max_pages)
    for t in (cache.k, cache.v):
        t.copy_(torch.as_tensor(rng.normal(size=t.shape).astype(np.float32)))
    return cache


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 4), (7, 1), (28, 4), (6, 3)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("page", [32, 128])
def test_store(hd, H, Hkv, f32, page):
    require_gpu()
    rng = np.random.default_rng(hd + H + page)
    B, max_pages, n_pages, rows, layer = 6, 8, 40, 150, 1
    cache = filled(2, n_pages, Hkv, hd, page, B, max_pages, rng)
    chunk = Chunk(B, rows)
    first = np.array([5, 0, 31, 8, 64, 1])
    put(chunk.count, np.where(first > 0, first, 0))
    cache_plan(cache, chunk, reset=True)
    count = np.array([1, 40, 33, 8, 0, 7])             # single tokens, whole and partial runs of 8
    put(chunk.start, first); put(chunk.count, count)
    cache_plan(cache, chunk)
    T = int(count.sum())
    k0, v0 = cache.k.clone(), cache.v.clone()
    width = (H + 2 * Hkv) * hd
    buf = torch.as_tensor(rng.normal(size=(rows, width + 8)).astype(np.float32)).cuda()
    x = (buf if f32 else buf.to(torch.bfloat16))[:, :width]
    rope = rope_table(200, hd, 1e4)
    q = torch.full((rows, H, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    cache_store(cache, layer, x, H, chunk, rope=rope, q=q)
    pos, slots = chunk.positions[:T].cpu().long(), chunk.slots[:T].cpu().long()
    xx = x[:T].double().cpu().reshape(T, H + 2 * Hkv, hd)
    cs = rope.double().cpu()[pos]
    a, b = xx[:, :H + Hkv, :hd // 2], xx[:, :H + Hkv, hd // 2:]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    want = torch.cat([a * c - b * s, b * c + a * s], -1)
    # two products and a sum in fp32 (2^-24 each of the magnitudes), one rounding to bf16 (2^-8)
    mag = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)
    tol = 2.0 ** -8 * want.abs() + 3 * 2.0 ** -24 * mag * (1 + 2.0 ** -8)
    got_q = q[:T].double().cpu()
    assert ((got_q - want[:, :H]).abs() <= tol[:, :H]).all()
    assert (q[T:] == 7).all()
    ko, vo = ref.offsets(page, hd)
    kn, vn = (ref.natural(t[layer], o).cpu() for t, o in ((cache.k, ko), (cache.v, vo)))
    got_k = kn[slots // page, :, slots % page].double()
    assert ((got_k - want[:, H:]).abs() <= tol[:, H:]).all()
    assert torch.equal(vn[slots // page, :, slots % page], xx[:, H + Hkv:].to(torch.bfloat16))
    # everything else as it was
    for t, t0, o in ((cache.k, k0, ko), (cache.v, v0, vo)):
        assert torch.equal(t[0], t0[0])
        n, n0 = ref.natural(t[layer], o).cpu(), ref.natural(t0[layer], o).cpu()
        n[slots // page, :, slots % page] = 0
        n0[slots // page, :, slots % page] = 0
        assert torch.equal(n, n0)


def test_store_leaves_bad_rows_out():
    require_gpu()
    rng = np.random.default_rng(2)
    hd, H, page = 64, 2, 32
    cache = filled(1, 3, H, hd, page, 1, 3, rng)
    k0, v0 = cache.k.clone(), cache.v.clone()
    chunk = Chunk(1, 6)
    put(chunk.cu, [0, 6])
    put(chunk.positions, [0, 5, -1, 50, 3, 1 << 30])   # the table has 40 positions
    put(chunk.slots, [-1, 96, 4, 5, 7, 8])             # the cache 96 slots
    x = torch.as_tensor(rng.normal(size=(6, 3 * H * hd)).astype(np.float32)).cuda().to(torch.bfloat16)
    q = cache_store(cache, 0, x, H, chunk, rope=rope_table(40, hd, 1e4))
    torch.cuda.synchronize()
    live = [4]
    assert (q[[0, 1, 2, 3, 5]] == 0).all() and (q[live] != 0).any()
    kn, kn0 = (ref.natural(t[0], ref.offsets(page, hd)[0]) for t in (cache.k, k0))
    assert not torch.equal(kn[0, :, 7], kn0[0, :, 7])
    kn[0, :, 7] = 0; kn0[0, :, 7] = 0
    assert torch.equal(kn, kn0)
    vn, vn0 = (ref.natural(t[0], ref.offsets(page, hd)[1]) for t in (cache.v, v0))
    vn[0, :, 7] = 0; vn0[0, :, 7] = 0
    assert torch.equal(vn, vn0)


def test_store_without_rotation_or_q():
    require_gpu()
    rng = np.random.default_rng(4)
    hd, H, page = 128, 3, 64
    cache = filled(1, 2, H, hd, page, 1, 2, rng)
    chunk = Chunk(1, 70)
    put(chunk.count, [70])
    cache_plan(cache, chunk, reset=True)
    x = torch.as_tensor(rng.normal(size=(70, 3 * H * hd)).astype(np.float32)).cuda().to(torch.bfloat16)
    q = cache_store(cache, 0, x, H, chunk)
    xx = x.view(70, 3 * H, hd)
    assert torch.equal(q, xx[:, :H])
    sl = chunk.slots.long()
    for t, o, lo in ((cache.k, ref.offsets(page, hd)[0], H), (cache.v, ref.offsets(page, hd)[1], 2 * H)):
        assert torch.equal(ref.natural(t[0], o)[sl // page, :, sl % page], xx[:, lo:lo + H])


def test_rope_table_far_out():
    """Angles of far positions come from 64 bits: the table is within an fp32 rounding of them."""
    require_gpu()
    t = rope_table(300001, 64, 1e4)[-1].double().cpu().numpy()
    ang = 300000.0 * 1e4 ** (-2.0 * np.arange(32) / 64)
    assert np.abs(t - np.stack([np.cos(ang), np.sin(ang)], -1)).max() <= 2.0 ** -24


# ---- attention -----------------------------------------------------------------------------------
def requests(rng, lens, count, hd, H, Hkv, page, spare=3, rows=None, garbage=math.nan, layers=1):
    """A cache whose requests hold `lens` keys in pages of random order, everything behind them
    garbage; chunks of the last `count` positions; natural K and V of each request."""
    B = len(lens)
    lens, count = np.asarray(lens), np.asarray(count)
    need = -(-lens // page)
    n_pages, max_pages = int(need.sum()) + spare, int(max(1, need.max()))
    cache = KVCache(layers, n_pages, Hkv, hd, page, B, max_pages)
    order = rng.permutation(n_pages)
    table, at = np.full((B, max_pages), -1), 0
    kn = torch.full((n_pages, Hkv, page, hd), garbage, dtype=torch.bfloat16)
    vn = kn.clone()
    ks, vs = [], []
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        k, v = (torch.as_tensor(rng.normal(size=(lens[b], Hkv, hd)).astype(np.float32)).to(torch.bfloat16)
                for _ in range(2))
        for j in range(need[b]):
            n = min(page, lens[b] - j * page)
            kn[table[b, j], :, :n] = k[j * page:j * page + n].transpose(0, 1)
            vn[table[b, j], :, :n] = v[j * page:j * page + n].transpose(0, 1)
        ks.append(k.double().cuda())
        vs.append(v.double().cuda())
    ko, vo = ref.offsets(page, hd)
    cache.k[layers - 1].copy_(ref.operand(kn, ko))
    cache.v[layers - 1].copy_(ref.operand(vn, vo))
    put(cache.table, table); put(cache.len, lens)
    T = int(count.sum())
    chunk = Chunk(B, rows or max(1, T))
    put(chunk.start, lens - count); put(chunk.count, count)
    put(chunk.cu, np.concatenate([[0], np.cumsum(count)]))
    q = torch.as_tensor(rng.normal(size=(chunk.rows, H, hd)).astype(np.float32)).to(torch.bfloat16).cuda()
    return cache, chunk, q, ks, vs, T


def compare(cache, chunk, q, ks, vs, T, causal, layer=0, scale=None, lens=None, **kw):
    out = torch.full_like(q, 9.0)
    cache_attention(cache, layer, q, chunk, causal=causal, out=out, scale=scale, **kw)
    lens = cache.len.cpu().tolist() if lens is None else lens
    want, mag, dev = ref.attend(q[:T].double(), ks, vs, lens, chunk.start.cpu().tolist(),
                                chunk.cu.cpu().tolist(), q.shape[1] // cache.n_kv_heads, causal,
                                cache.head_dim ** -0.5 if scale is None else scale)
    err = (out[:T].double() - want).abs()
    tol = ref.attend_tolerance(want, mag, dev)
    assert not torch.isnan(out[:T]).any()
    assert (err <= tol).all(), (float((err / tol).max()),)
    assert (out[T:] == 9).all()
    return out


HEADS = [(1, 1), (4, 4), (7, 1), (28, 4), (8, 2), (3, 3), (32, 2)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("page", [32, 64, 256])
def test_attention_single_tokens(hd, H, Hkv, causal, page):
    require_gpu()
    rng = np.random.default_rng(hd + H + page)
    lens = [1, 2, 31, 32, 33, 63, 64, 65, 100, 257, 1000, 5]
    log_case(f"tokens hd={hd} H={H}/{Hkv} page={page} causal={causal}")
    compare(*requests(rng, lens, [1] * len(lens), hd, H, Hkv, page), causal)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_chunks(hd, H, Hkv, causal):
    """Ragged chunks, among them empty ones and whole sequences; rows behind the last one."""
    require_gpu()
    rng = np.random.default_rng(100 + hd + H)
    lens = [130, 70, 64, 1, 200, 33, 96, 500]
    count = [17, 0, 64, 1, 5, 33, 32, 100]
    log_case(f"chunks hd={hd} H={H}/{Hkv} causal={causal}")
    args = requests(rng, lens, count, hd, H, Hkv, 64, rows=sum(count) + 37)
    compare(*args, causal)


@pytest.mark.parametrize("max_count", [1, 3, 20, 70, 0])
@pytest.mark.parametrize("max_len", [1, 300, 5000, 0])
@pytest.mark.parametrize("hd,H,Hkv", [(128, 8, 2), (64, 2, 2)])
def test_attention_whatever_was_expected(max_count, max_len, hd, H, Hkv):
    """Every kernel and split on the same requests, whether or not they fit what was expected."""
    require_gpu()
    rng = np.random.default_rng(7)
    lens, count = [900, 40, 2100, 64, 1], [40, 1, 9, 64, 1]
    for causal in (False, True):
        args = requests(rng, lens, count, hd, H, Hkv, 32)
        compare(*args, causal, max_count=max_count, max_len=max_len)


@pytest.mark.parametrize("B", [1, 63, 64, 65, 130, 700])
def test_attention_many_requests(B):
    require_gpu()
    rng = np.random.default_rng(B)
    lens = rng.integers(1, 90, size=B)
    count = np.minimum(lens, rng.integers(0, 6, size=B))
    if count.sum() == 0:
        count[0] = 1
    compare(*requests(rng, lens, count, 64, 4, 2, 32), True, max_count=5, max_len=90)


@pytest.mark.parametrize("causal", [False, True])
def test_attention_long_prompt(causal):
    """Tiles of 128 rows over many key tiles, and a chunk that ends inside one."""
    require_gpu()
    rng = np.random.default_rng(3)
    compare(*requests(rng, [1500, 700], [1100, 333], 128, 4, 2, 128), causal)


def test_attention_far_pages():
    """Element offsets past 2^31 in the pool."""
    require_gpu()
    rng = np.random.default_rng(5)
    hd, H, page = 128, 2, 256
    n_pages = 2 ** 31 // (H * page * hd) + 50            # 2^31 elements and some more
    cache = KVCache(1, n_pages, H, hd, page, 1, 4)
    chunk = Chunk(1, 600)
    put(chunk.count, [600])
    put(cache.free, np.arange(n_pages))                  # the last pages are handed out first
    cache_plan(cache, chunk)
    x = torch.as_tensor(rng.normal(size=(600, 3 * H * hd)).astype(np.float32)).cuda().to(torch.bfloat16)
    assert int(chunk.slots.max()) // page == n_pages - 1
    q = cache_store(cache, 0, x, H, chunk)
    xx = x.view(600, 3, H, hd).double()
    compare(cache, chunk, q, [xx[:, 1]], [xx[:, 2]], 600, False)


def test_attention_in_the_middle_of_a_sequence():
    """A chunk that is followed by cached keys: both directions see them, causal rows do not."""
    require_gpu()
    rng = np.random.default_rng(6)
    for causal in (False, True):
        args = requests(rng, [300, 90], [20, 8], 64, 4, 4, 32)
        put(args[1].start, [100, 0])
        compare(*args, causal)


def test_rows_without_a_key_are_zero():
    require_gpu()
    rng = np.random.default_rng(9)
    for count in ([3, 2], [200, 2]):                       # both kernels
        cache, chunk, q, ks, vs, T = requests(rng, [max(count), 40], count, 64, 2, 1, 32)
        put(cache.len, [0, 40])
        for max_len in (0, 10):
            out = compare(cache, chunk, q, ks, vs, T, False, max_len=max_len)
            assert (out[:count[0]] == 0).all()
        put(chunk.start, [-500, 38])                       # causal rows before position 0
        put(cache.len, [max(count), 40])
        out = torch.full_like(q, 9.0)
        cache_attention(cache, 0, q, chunk, causal=True, out=out)
        assert (out[:count[0]] == 0).all() and not torch.isnan(out).any()


@pytest.mark.parametrize("gain", [1e-3, 1.0, 30.0])
def test_attention_scores_of_any_size(gain):
    """Peaked and flat rows; a reference maximum that moves late."""
    require_gpu()
    rng = np.random.default_rng(13)
    args = list(requests(rng, [1200, 77], [9, 40], 128, 4, 4, 64))
    args[2] = (args[2].float() * gain).to(torch.bfloat16)
    compare(*args, True)
    compare(*args, False, scale=0.01)


def test_non_finite_keys_and_values_reach_only_rows_that_see_them():
    require_gpu()
    rng = np.random.default_rng(14)
    for n, c in ((100, 10), (400, 300)):                   # both kernels
        cache, chunk, q, ks, vs, T = requests(rng, [n], [c], 64, 1, 1, 32)
        bad = n - c + c // 2                               # the position of the middle row
        page = int(cache.table[0, bad // 32])
        ko, vo = ref.offsets(32, 64)
        clean = torch.full_like(q, 9.0)
        cache_attention(cache, 0, q, chunk, causal=True, out=clean)
        for t, o in ((cache.k, ko), (cache.v, vo)):
            for value in (math.nan, math.inf):
                was = t.clone()
                t[0, page, 0, o[bad % 32]] = value
                out = torch.full_like(q, 9.0)
                cache_attention(cache, 0, q, chunk, causal=True, out=out)
                assert torch.equal(out[:c // 2], clean[:c // 2])
                assert torch.isnan(out[c // 2:].float()).any(dim=-1).all() or value == math.inf
                t.copy_(was)


def test_layers_streams_graph_and_workspaces():
    require_gpu()
    rng = np.random.default_rng(15)
    cache, chunk, q, ks, vs, T = requests(rng, [3000, 500, 2000], [1, 1, 1], 128, 4, 2, 64, layers=3)
    kw = dict(max_count=1, max_len=3000)
    n = cache_attention_workspace(cache, 4, chunk, 1, 3000)
    assert n > 0
    want = compare(cache, chunk, q, ks, vs, T, True, layer=2, **kw)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [cache_attention(cache, 2, q, chunk, causal=True, stream=s, **kw) for s in streams]
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    cache_attention(cache, 2, q, chunk, causal=True, out=out, workspace=ws, **kw)
    torch.cuda.synchronize()
    for o in outs + [out]:
        assert torch.equal(o, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache_attention(cache, 2, q, chunk, causal=True, out=out, workspace=ws, **kw)
    for lens in ([3000, 500, 2000], [10, 64, 1], [1, 500, 1999]):
        put(cache.len, lens); put(chunk.start, np.array(lens) - 1)
        q.copy_(torch.as_tensor(rng.normal(size=q.shape).astype(np.float32)))
        ws.fill_(255)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, compare(cache, chunk, q, ks, vs, T, True, layer=2, **kw))


def test_a_rows_sums_do_not_depend_on_its_batch():
    """The same request alone and beside others, with the sizes of the larger batch expected."""
    require_gpu()
    rng = np.random.default_rng(16)
    cache, chunk, q, ks, vs, T = requests(rng, [700, 90, 1500], [12, 3, 1], 128, 8, 2, 64)
    kw = dict(max_count=12, max_len=1500, causal=True)
    all_rows = cache_attention(cache, 0, q, chunk, **kw)
    put(chunk.count, [12, 0, 0]); put(chunk.cu, [0, 12, 12, 12])
    alone = cache_attention(cache, 0, q, chunk, out=torch.zeros_like(q), **kw)
    assert torch.equal(alone[:12], all_rows[:12])


def test_refusals():
    require_gpu()
    rng = np.random.default_rng(17)
    cache, chunk, q, ks, vs, T = requests(rng, [3000, 500], [1, 1], 64, 4, 2, 64)
    with pytest.raises(CoraError, match="workspace"):
        cache_attention(cache, 0, q, chunk, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"),
                        max_count=1, max_len=3000)
    with pytest.raises(CoraError, match="scale"):
        cache_attention(cache, 0, q, chunk, scale=0.0)
    with pytest.raises(CoraError, match="layer"):
        cache_attention(cache, 1, q, chunk)
    with pytest.raises(CoraError, match="multiple"):
        cache_attention(cache, 0, q[:, :3].contiguous(), chunk)
    with pytest.raises(ValueError, match="q"):
        cache_attention(cache, 0, q[:1].contiguous(), chunk)
    with pytest.raises(ValueError, match="contiguous"):
        cache_attention(cache, 0, q.transpose(0, 1), chunk)
    with pytest.raises(ValueError, match="requests"):
        cache_plan(cache, Chunk(3, 4))
    x = torch.zeros((2, 8 * 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="x"):
        cache_store(cache, 0, x[:, 1:], 4, chunk)
    with pytest.raises(ValueError, match="rope"):
        cache_store(cache, 0, x, 4, chunk, rope=torch.zeros((5, 64, 2), device="cuda"))
    bad = torch.zeros((2, 8 * 64 + 4), dtype=torch.bfloat16, device="cuda")[:, :8 * 64]
    with pytest.raises(CoraError, match="aligned"):
        cache_store(cache, 0, bad, 4, chunk)
