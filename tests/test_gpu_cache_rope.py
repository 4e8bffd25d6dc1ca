"""cache_store's table of angles: what is not a table of at least one position is refused."""
import pytest
import torch

from paper_2608_11235_amd import Chunk, KVCache, cache_plan, cache_store, rope_table
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


def test_tables_that_are_refused():
    """An empty table has no address, which the library would take for rows already rotated."""
    require_gpu()
    cache, chunk = KVCache(1, 2, 1, 64, 32, 1, 2), Chunk(1, 4)
    chunk.count.fill_(4)
    cache_plan(cache, chunk)
    cache.k.zero_()
    x = torch.ones((4, 3 * 64), dtype=torch.bfloat16, device="cuda")
    for bad, error in ((rope_table(0, 64, 1e4), ValueError), (rope_table(8, 128, 1e4), ValueError),
                       (rope_table(8, 64, 1e4)[0], ValueError), (rope_table(8, 64, 1e4).double(), TypeError),
                       (rope_table(8, 64, 1e4, device="cpu"), ValueError), ([1.0], TypeError)):
        with pytest.raises(error, match="rope"):
            cache_store(cache, 0, x, 1, chunk, rope=bad)
    torch.cuda.synchronize()
    assert (cache.k == 0).all()
    cache_store(cache, 0, x, 1, chunk, rope=rope_table(4, 64, 1e4))
    assert (cache.k != 0).any()
