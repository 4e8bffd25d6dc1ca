"""Chunks without a row: a capacity of 0 is a chunk like any other, whose arrays may be null."""
import numpy as np
import pytest
import torch

from paper_2608_11235_amd import Chunk, Model, cache_attention, cache_plan, cache_store
from tests.gpu_common import require_gpu
from tests.test_cache_abi import INVALID, UNSUPPORTED, attend, cache, chunk, lib, pages, store  # noqa: F401


def test_store_and_attention_do_nothing(lib):  # noqa: F811
    none = chunk(lib, rows=0)
    assert store(lib, ch=none, x=None, q=None, rope=None) == 0
    assert attend(lib, ch=none, q=None, out=None, ws=None, n=0) == 0
    # what describes the cache is still checked
    assert store(lib, ch=none, x=None, layer=2) == INVALID
    assert store(lib, ch=none, x=None, ca=cache(lib, head_dim=96)) == UNSUPPORTED
    assert attend(lib, ch=none, q=None, heads=5) == UNSUPPORTED
    assert attend(lib, ch=none, q=None, pg=pages(lib, n_pages=7)) == INVALID


@pytest.mark.gpu
def test_a_pass_without_rows():
    """Through the binding, where an empty tensor has no address: pages are given back, and the store,
    the attention and the cached pass leave everything as it was."""
    require_gpu()
    from tests.test_gpu_cached_pass import HD128, cache_for, put
    spec = HD128
    kv, first, none = cache_for(spec, 2, 64), Chunk(2, 40), Chunk(2, 0)
    put(first.count, [30, 10])
    cache_plan(kv, first)
    put(none.start, [30, 10]); put(none.count, [-1, 0])
    cache_plan(kv, none)
    assert kv.len.tolist() == [0, 10] and none.cu.tolist() == [0, 0, 0] and none.status.tolist() == [0, 0]
    put(none.count, [1, 1])
    put(none.start, [0, 10])
    cache_plan(kv, none)                               # no room for a row
    assert kv.len.tolist() == [0, 10] and none.status.tolist() == [UNSUPPORTED, UNSUPPORTED]
    kv.k.zero_(); kv.v.zero_()
    hd, H = spec.head_dim, spec.n_heads
    x = torch.empty((0, (H + 2 * spec.n_kv_heads) * hd), dtype=torch.bfloat16, device="cuda")
    q = cache_store(kv, 1, x, H, none)
    assert q.shape == (0, H, hd)
    for kw in ({}, {"max_count": 1, "max_len": 5000}):
        assert cache_attention(kv, 1, q, none, **kw).shape == (0, H, hd)
    with Model(spec, 0, 1, 64) as m:
        out = m.forward_cached(kv, none, torch.empty(0, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert out.shape == (0, spec.vocab) and (kv.k == 0).all() and (kv.v == 0).all()
    assert np.array_equal(kv.len.cpu().numpy(), [0, 10])
