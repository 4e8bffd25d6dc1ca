"""Requests that go on as their parents: tables, counts, stack and copies equal the host's, and every request's
K and V are what its history stored."""
import numpy as np
import pytest
import torch

from paper_2608_11235_amd import (Chunk, KVCache, cache_attention, cache_plan, cache_reorder, cache_store, quantize_rows,
                                  rows8_product, vocab_beam)
from tests.cache_ref import natural, offsets
from tests.gpu_common import log_case, require_gpu
from tests.reorder_ref import SharedPlan

pytestmark = pytest.mark.gpu


def put(t, a):
    t.copy_(torch.as_tensor(np.asarray(a), dtype=t.dtype))


def agree(cache, host):
    n = len(host.free)
    assert cache.len.cpu().tolist() == host.len.tolist()
    assert int(cache.n_free) == n and cache.free[:n].cpu().tolist() == host.free
    assert cache.refs.cpu().tolist() == host.refs.tolist()
    table = cache.table.cpu().numpy()
    for b in range(host.B):
        assert [int(x) for x in table[b, :len(host.held(b))]] == host.held(b), b
    # what is neither free nor held is nobody's: all pages are one or the other
    assert sorted(host.free + [p for p in range(host.n_pages) if host.refs[p] > 0]) == list(range(host.n_pages))


class Search:
    """A cache under test beside its host model, whose requests' histories are lists of token numbers; the K and V of
    token t in layer l hold t and l."""

    def __init__(self, batch, max_pages, n_pages, page, layers=2, heads=2, hd=64):
        self.cache = KVCache(layers, n_pages, heads, hd, page, batch, max_pages, shared=True)
        self.host = SharedPlan(batch, max_pages, n_pages, page)
        self.story = [[] for _ in range(batch)]
        self.next, self.page, self.hd, self.heads, self.layers, self.B = 1, page, hd, heads, layers, batch

    def value(self, t, layer):
        """bf16 rows of a token: numbers of 7 bits that say which it is."""
        t = torch.as_tensor(t, dtype=torch.int64)
        j = torch.arange(self.heads * self.hd)
        return ((t[:, None] // 128 ** (j % 3)) % 128 + layer).to(torch.bfloat16).cuda()

    def plan(self, start, count, rows):
        chunk = Chunk(self.B, rows)
        put(chunk.start, start)
        put(chunk.count, count)
        cache_plan(self.cache, chunk)
        want = self.host.step(start, count, rows)
        assert chunk.status.cpu().tolist() == list(want["status"])
        assert chunk.cu.cpu().tolist() == want["cu"] and chunk.slots.cpu().tolist() == list(want["slots"])
        tokens = np.zeros(rows, np.int64)
        for b in range(self.B):
            if count[b] < 0:
                self.story[b] = []
            lo, hi = want["cu"][b], want["cu"][b + 1]
            if hi > lo:
                tokens[lo:hi] = np.arange(self.next, self.next + hi - lo)
                s = int(start[b])
                self.story[b][s:s + hi - lo] = list(tokens[lo:hi])
                self.next += hi - lo
        for layer in range(self.layers):
            x = self.value(tokens, layer)
            cache_store(self.cache, layer, torch.cat([x, x, -x], 1), self.heads, chunk)
        agree(self.cache, self.host)
        return want["status"]

    def reorder(self, parent):
        p = torch.as_tensor(np.asarray(parent), dtype=torch.int32).cuda()
        moves = torch.full((1 + 3 * self.B,), -9, dtype=torch.int32, device="cuda")
        status = cache_reorder(self.cache, p, moves=moves)
        want = self.host.reorder(parent)
        assert status.cpu().tolist() == want.tolist()
        agree(self.cache, self.host)
        m = moves.cpu().tolist()
        assert m[0] == len(self.host.moves)
        assert [tuple(m[1 + 3 * i:4 + 3 * i]) for i in range(m[0])] == self.host.moves
        assert all(x == -9 for x in m[1 + 3 * m[0]:])
        old = [list(x) for x in self.story]
        ok = [b if not -1 <= parent[b] < self.B else (-1 if want[b] == -3 else int(parent[b])) for b in range(self.B)]
        self.story = [old[q] if q >= 0 else [] for q in ok]
        self.story = [list(x) for x in self.story]
        return want

    def check(self):
        """Every request reads its own history."""
        ko, vo = offsets(self.page, self.hd)
        k, v = natural(self.cache.k, ko), natural(self.cache.v, vo)   # [layers, pages, heads, page, hd]
        for b in range(self.B):
            n = len(self.story[b])
            assert n == int(self.host.len[b])
            if n == 0:
                continue
            pages = torch.as_tensor(self.host.held(b)).cuda()
            for layer in range(self.layers):
                want = self.value(self.story[b], layer).view(n, self.heads, self.hd)
                for got, sign in ((k, 1), (v, -1)):
                    g = got[layer, pages].transpose(1, 2).reshape(-1, self.heads, self.hd)[:n]
                    assert torch.equal(g, sign * want), (b, layer)


@pytest.mark.parametrize("page,hd,heads", [(32, 64, 2), (64, 128, 1), (128, 64, 3), (256, 128, 2)])
def test_a_search(page, hd, heads):
    """Prompts into every beam of a request, then tokens and reorders, a release and a new prompt on the way."""
    require_gpu()
    log_case(f"search page {page} hd {hd} heads {heads}")
    rng = np.random.default_rng(page + hd)
    s = Search(8, 4, 30, page, heads=heads, hd=hd)
    prompts = [int(page * 1.5), 0, 0, 0, page, 0, 0, 0]
    s.plan([0] * 8, prompts, 3 * page)
    s.reorder([0, 0, 0, 0, 4, 4, 4, 4])
    s.check()
    for step in range(12):
        n = int(rng.integers(1, 4))
        s.plan(s.host.len.tolist(), [n] * 8, 8 * n)
        parent = np.concatenate([rng.integers(0, 4, size=4), 4 + rng.integers(0, 4, size=4)])
        if step == 5:
            parent[2] = -1
        if step == 8:
            parent[[1, 6]] = [8, -2]
        s.reorder(parent.tolist())
        s.check()
        if step == 9:
            s.plan(s.host.len.tolist(), [-1] * 4 + [0] * 4, 8)
            s.plan([0] * 8, [page + 7, 0, 0, 0, 0, 0, 0, 0], 2 * page)
            s.reorder([0, 0, 0, 0, 7, 6, 5, 4])
            s.check()


def test_random_calls():
    """Any parents, releases, chunks inside shared pages, pools that run out."""
    require_gpu()
    rng = np.random.default_rng(11)
    seen = set()
    for B, most, pool in ((1, 3, 3), (3, 4, 6), (7, 3, 14), (20, 5, 40), (33, 2, 40)):
        log_case(f"random calls, {B} requests, {pool} pages")
        s = Search(B, most, pool, 32, layers=1)
        for step in range(25):
            kind = rng.random()
            if kind < 0.55:
                count = rng.integers(-1, 25, size=B) * (rng.random(B) < 0.7)
                start = np.maximum(s.host.len - (rng.random(B) < 0.3) * rng.integers(0, 40, size=B), 0)
                seen |= set(s.plan(np.where(count < 0, 0, start).tolist(), count.tolist(), int(rng.integers(1, 20 * B))))
            else:
                parent = rng.integers(0, B, size=B)
                parent[rng.random(B) < 0.2] = -1
                parent[rng.random(B) < 0.05] = B + 3
                seen |= set(s.reorder(parent.tolist()))
            s.check()
    assert {-5, -3, -2, -1, 0} <= {int(x) for x in seen}, seen


@pytest.mark.parametrize("B", [1, 2, 1023, 1025, 4096])
def test_many_requests(B):
    """More requests than threads; rows of tables that several passes write."""
    require_gpu()
    log_case(f"reorder {B} requests")
    rng = np.random.default_rng(B)
    s = Search(B, 5, 4 * B + 8, 32, layers=1, heads=1)
    n = rng.integers(0, 90, size=B)
    s.plan([0] * B, n.tolist(), int(n.sum()) + 3)
    for parent in (rng.integers(0, B, size=B), rng.permutation(B), np.arange(B)):
        s.reorder(parent.tolist())
    s.check()


def test_long_tables():
    require_gpu()
    log_case("reorder long tables")
    s = Search(3, 700, 2300, 32, layers=1, heads=1)
    s.plan([0, 0, 0], [700 * 32, 20001, 17], 43000)
    s.reorder([1, 0, 1])
    s.reorder([1, 2, -1])
    s.check()


def test_no_page_left_for_a_copy():
    """The beams in front get the pages that are there, the others become empty; their parents keep theirs."""
    require_gpu()
    log_case("reorder without pages")
    s = Search(6, 3, 5, 32)
    s.plan([0] * 6, [70, 0, 0, 0, 0, 0], 70)
    assert s.reorder([0, 0, 0, 0, 0, 0]).tolist() == [0, 0, 0, -3, -3, -3]
    s.check()
    assert s.reorder([1, 1, 2, 3, 0, 0]).tolist() == [0, -3, 0, 0, 0, -3]
    s.check()
    s.plan(s.host.len.tolist(), [-1, -1, -1, 0, 0, -1], 8)
    s.check()


def test_a_chunk_in_a_shared_page_is_refused():
    require_gpu()
    log_case("chunk in a shared page")
    s = Search(3, 4, 12, 32)
    s.plan([0, 0, 0], [50, 0, 10], 64)
    s.reorder([0, 0, 2])
    assert list(s.plan([31, 32, 0], [10, 10, 5], 64)) == [-5, 0, 0]
    s.check()
    assert list(s.plan([0, 20, 10], [40, 5, 3], 64)) == [-5, -5, 0]
    s.plan([0, 0, 0], [0, -1, 0], 64)
    assert list(s.plan([0, 0, 0], [40, 0, 0], 64)) == [0, 0, 0]     # alone again
    s.check()


def test_reset_forgets_the_holders():
    require_gpu()
    s = Search(2, 4, 8, 32)
    s.plan([0, 0], [60, 0], 64)
    s.reorder([0, 0])
    chunk = Chunk(2, 64)
    put(chunk.count, [40, 0])
    cache_plan(s.cache, chunk, reset=True)
    s.host.step([0, 0], [40, 0], 64, reset=True)
    agree(s.cache, s.host)


def test_a_page_of_nonsense_is_left_alone():
    """Entries that are no pages of the pool: neither counts nor pages outside it are touched."""
    require_gpu()
    log_case("nonsense pages")
    s = Search(4, 3, 8, 32)
    s.plan([0] * 4, [70, 40, 10, 0], 128)
    s.cache.table[0, 1] = 1 << 30
    s.cache.table[1, 1] = -7
    k = s.cache.k.clone()
    status = cache_reorder(s.cache, torch.tensor([0, 0, 1, 1], dtype=torch.int32, device="cuda"))
    assert status.tolist() == [0, 0, 0, 0]
    refs, n = s.cache.refs.cpu().tolist(), int(s.cache.n_free)
    assert all(0 <= r <= 4 for r in refs) and 0 <= n <= 8
    changed = (s.cache.k != k).flatten(2).any(2).any(0)
    assert int(changed.sum()) <= 2


def test_graph_streams():
    """Plan, reorder and their pages captured once and replayed as the parents change."""
    require_gpu()
    log_case("reorder graph")
    rng = np.random.default_rng(3)
    a, b = (Search(6, 6, 30, 32) for _ in range(2))
    for s in (a, b):
        s.plan([0] * 6, [40, 0, 0, 33, 0, 0], 80)
    parent = torch.tensor([0, 0, 0, 3, 3, 3], dtype=torch.int32, device="cuda")
    status = torch.zeros(6, dtype=torch.int32, device="cuda")
    moves = torch.zeros(19, dtype=torch.int32, device="cuda")
    chunk = Chunk(6, 6)
    chunk.count.fill_(1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache_reorder(a.cache, parent, status=status, moves=moves)
        chunk.start.copy_(a.cache.len)
        cache_plan(a.cache, chunk)
    side = torch.cuda.Stream()
    for rep in range(6):
        g.replay()
        torch.cuda.synchronize()
        other = Chunk(6, 6)
        other.count.fill_(1)
        side.wait_stream(torch.cuda.default_stream())
        st = cache_reorder(b.cache, parent, stream=side)
        with torch.cuda.stream(side):
            other.start.copy_(b.cache.len)
            cache_plan(b.cache, other)
        torch.cuda.synchronize()
        for name in ("table", "len", "refs", "n_free"):
            assert torch.equal(getattr(a.cache, name), getattr(b.cache, name)), (rep, name)
        n = int(a.cache.n_free)
        assert torch.equal(a.cache.free[:n], b.cache.free[:n])
        assert torch.equal(status, st) and torch.equal(chunk.slots, other.slots)
        put(parent, np.concatenate([rng.integers(0, 3, 3), 3 + rng.integers(0, 3, 3)]))


def test_decode_with_beams_equals_one_request_each():
    """8-bit logits, beams, reorder, plan, store and attention together: what each beam attends to equals a cache that
    holds its history alone."""
    require_gpu()
    log_case("beams together")
    rng = np.random.default_rng(8)
    K, H, hd, V, page = 3, 2, 64, 500, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    emb = torch.randn((V, 3 * H * hd), generator=g, device="cuda").to(torch.bfloat16)
    head = quantize_rows(torch.randn((V, H * hd), generator=g, device="cuda") * 0.3)
    beams = KVCache(1, 40, H, hd, page, 2 * K, 8, shared=True)
    prompts = [rng.integers(0, V, 45).tolist(), rng.integers(0, V, 32).tolist()]
    first = Chunk(2 * K, 96)
    put(first.count, [45, 0, 0, 32, 0, 0])
    cache_plan(beams, first)
    x = torch.zeros((96, emb.shape[1]), dtype=torch.bfloat16, device="cuda")
    x[:77] = emb[torch.tensor(prompts[0] + prompts[1], device="cuda")]
    cache_store(beams, 0, x, H, first)
    cache_reorder(beams, torch.tensor([0, 0, 0, 3, 3, 3], dtype=torch.int32, device="cuda"))
    story = [list(prompts[b // K]) for b in range(2 * K)]
    token = torch.tensor([5, 6, 7, 8, 9, 10], dtype=torch.int32, device="cuda")
    score = torch.tensor([0.0, -1.0, -2.0] * 2, device="cuda")
    chunk = Chunk(2 * K, 2 * K)
    chunk.count.fill_(1)
    parents_seen = set()
    for step in range(40):
        chunk.start.copy_(beams.len)
        cache_plan(beams, chunk)
        assert chunk.status.tolist() == [0] * 2 * K
        for b, t in enumerate(token.tolist()):
            story[b].append(t)
        q = cache_store(beams, 0, emb[token.long()], H, chunk)
        out = cache_attention(beams, 0, q, chunk, max_count=1, max_len=256, causal=True)
        alone = KVCache(1, 8 * 2 * K, H, hd, page, 2 * K, 8)
        whole = Chunk(2 * K, sum(len(s) for s in story))
        put(whole.count, [len(s) for s in story])
        cache_plan(alone, whole)
        cache_store(alone, 0, emb[torch.tensor(sum(story, []), device="cuda")], H, whole)
        want = cache_attention(alone, 0, q, chunk, max_count=1, max_len=256, causal=True)
        assert torch.equal(out, want), step
        logits = rows8_product(quantize_rows(out.view(2 * K, -1)), head)
        tok, parent, score = vocab_beam(logits, K, V - 1, score.view(-1))
        assert (tok >= 0).all() and (parent.view(2, K) // K == torch.tensor([[0], [1]], device="cuda")).all()
        cache_reorder(beams, parent.view(-1))
        p = parent.view(-1).tolist()
        parents_seen.add(tuple(p))
        story = [list(story[q]) for q in p]
        token = tok.view(-1)
        score = score - score.amax(dim=1, keepdim=True)
    assert len(parents_seen) > 3


def test_refusals():
    require_gpu()
    ok = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="shared"):
        cache_reorder(KVCache(1, 4, 1, 64, 32, 2, 2), ok)
    cache = KVCache(1, 4, 1, 64, 32, 2, 2, shared=True)
    with pytest.raises(ValueError, match="parent"):
        cache_reorder(cache, ok[:1])
    with pytest.raises(TypeError, match="parent"):
        cache_reorder(cache, ok.long())
    with pytest.raises(ValueError, match="moves"):
        cache_reorder(cache, ok, moves=torch.zeros(6, dtype=torch.int32, device="cuda"))
    cache_reorder(cache, ok)
    assert cache.len.tolist() == [0, 0]
