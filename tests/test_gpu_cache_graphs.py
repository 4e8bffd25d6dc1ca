"""Cache attention's largest batch at its largest tile of few rows, and captured graphs whose
workspaces torch's allocator holds."""
import numpy as np
import pytest
import torch

from paper_2608_11235_amd import cache_attention, cache_attention_workspace
from tests.gpu_common import log_case, require_gpu
from tests.test_gpu_cache import compare, put, requests

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_count", [8, 16])
def test_largest_batch_of_wide_heads(max_count):
    """4096 requests, heads of 128, 16 and 32 rows a tile: the most shared memory a workgroup takes."""
    require_gpu()
    rng = np.random.default_rng(max_count)
    lens = rng.integers(1, 5, size=4096)
    lens[[0, 2000, 4095]] = [900, 33, 64]
    count = np.minimum(lens, rng.integers(0, 3, size=4096))
    count[[0, 2000]] = [16, 9]
    log_case(f"4096 requests of wide heads, max_count {max_count}")
    compare(*requests(rng, lens, count, 128, 2, 1, 32), True, max_count=max_count, max_len=900)


def test_two_graphs_at_once_without_a_given_workspace():
    """Each capture holds a workspace of its own: replays that overlap give what eager calls give."""
    require_gpu()
    rng = np.random.default_rng(3)
    sides = []
    for lens in ([4000, 700, 2500], [900, 5000, 64]):
        cache, chunk, q, *_ = requests(rng, lens, [1, 1, 1], 128, 8, 2, 64)
        kw = dict(max_count=1, max_len=max(lens), causal=True)
        assert cache_attention_workspace(cache, 8, chunk, 1, max(lens)) > 0
        out = torch.zeros_like(q)
        cache_attention(cache, 0, q, chunk, out=out, **kw)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            cache_attention(cache, 0, q, chunk, out=out, **kw)
        sides.append((cache, chunk, q, kw, out, g, torch.cuda.Stream()))
    for rep in range(4):
        for cache, chunk, q, *_ in sides:
            q.copy_(torch.as_tensor(rng.normal(size=q.shape).astype(np.float32)))
            put(chunk.start, cache.len.cpu().numpy() - 1)
        torch.cuda.synchronize()
        for *_, out, g, stream in sides:
            with torch.cuda.stream(stream):
                out.zero_()
                g.replay()
        torch.cuda.synchronize()
        for cache, chunk, q, kw, out, *_ in sides:
            assert torch.equal(out, cache_attention(cache, 0, q, chunk, **kw)), rep
