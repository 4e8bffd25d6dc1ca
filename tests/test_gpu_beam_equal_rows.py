"""Equal rows of beams have equal scores, so that ties go to the lowest beam."""
import pytest
import torch

from paper_2608_11235_amd import vocab_beam
from tests.gpu_common import log_case, require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [50, 2049, 50257])
def test_equal_rows_tie_wherever_they_lie(V):
    """One row at every alignment: the same scores to the last bit, so that the lowest beam has the first place."""
    require_gpu()
    log_case(f"equal rows V={V}")
    row = (2 * torch.randn(V, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda")).to(torch.bfloat16)
    for pitch in (V, V + 1, V + 3, V + 8):
        x = torch.full((64 * pitch + 8,), 90.0, dtype=torch.bfloat16, device="cuda")
        for start in (0, 1, 2, 5):
            rows = x[start:start + 64 * pitch].view(64, pitch)[:, :V]
            rows.copy_(row.expand(64, V))
            score = torch.full((64,), -1.5, device="cuda")
            token, parent, got = vocab_beam(rows, 8, 3, score, width=12)
            assert (parent[:, :8] == torch.arange(64, device="cuda").view(8, 8)).all() and (token[:, :8] == token[:, :1]).all()
            assert (got == got[0]).all() and (got[:, :8] == got[:, :1]).all()
