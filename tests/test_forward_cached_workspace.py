"""A workspace belongs to forward_cached on 8-bit weights: without them it is refused, not ignored."""
import pytest
import torch

import seeded_inputs as si
from paper_2608_11235_amd import Chunk, Model, cache_plan
from tests.gpu_common import log_case, require_gpu
from tests.test_gpu_cached_pass import cache_for, put


def test_refused_before_anything_else():
    class Held:
        pass
    with pytest.raises(ValueError, match="workspace"):
        Model.forward_cached(Held(), None, None, None, workspace=torch.zeros(4, dtype=torch.uint8))


@pytest.mark.gpu
def test_refused():
    require_gpu()
    log_case("workspace without weights")
    spec = si.TINY
    cache, chunk = cache_for(spec, 1, 64), Chunk(1, 16)
    put(chunk.count, [16])
    cache_plan(cache, chunk)
    tok = torch.zeros(16, dtype=torch.int32, device="cuda")
    with Model(spec, 0, 1, 64) as m:
        ws = torch.empty(m.quantized_workspace(16), dtype=torch.uint8, device="cuda")
        with pytest.raises(ValueError, match="workspace"):
            m.forward_cached(cache, chunk, tok, workspace=ws)
        m.forward_cached(cache, chunk, tok, workspace=ws, weights=m.quantize())
        m.forward_cached(cache, chunk, tok)
        torch.cuda.synchronize()
