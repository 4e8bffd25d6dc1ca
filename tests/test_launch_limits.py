"""Sizes beyond what one launch can count are refused on the host, not by the runtime (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2608_11235_amd import api
from tests.test_cache_abi import FAKE, UNSUPPORTED, attend, cache, chunk, lib, pages, store  # noqa: F401


@pytest.mark.parametrize("R", [1 << 23, (1 << 31) - 1])
def test_vocab_sample_rows(lib, R):  # noqa: F811
    rows = lib.SampleRows(temperature=FAKE, u=FAKE)
    assert lib.load().cora_vocab_sample(FAKE, R, 8, 8, 0, ctypes.byref(rows), FAKE, FAKE, None) == UNSUPPORTED


def test_vocab_gate_sampled_rows(lib):  # noqa: F811
    rows = lib.SampleRows(temperature=FAKE, u=FAKE)
    n = 1 << 18
    st = lib.State(*([FAKE] * 11), 33, 0, n)
    sc, gt = lib.SchedCfg(256, 32, 0, 0), lib.GateCfg(0.5, 1, 1, 0)
    assert lib.load().cora_vocab_gate_sampled(FAKE, n, 0, 8, 0, ctypes.byref(st), -1, ctypes.byref(sc),
                                              ctypes.byref(gt), ctypes.byref(rows), None) == UNSUPPORTED


@pytest.mark.parametrize("hd,heads", [(64, 1), (128, 1), (64, 4)])
def test_store_rows(lib, hd, heads):  # noqa: F811
    ca = cache(lib, head_dim=hd, n_kv_heads=heads)
    assert store(lib, ca=ca, ch=chunk(lib, rows=1 << 28), heads=heads, ld=3 * heads * hd) == UNSUPPORTED


def test_attention_workspace_of_many_rows(lib):  # noqa: F811
    """Where the merge of key ranges would exceed a launch, no range is split; the longest length
    that a call can name is as good as any beyond the tables."""
    f, n, m = lib.load().cora_cache_attention_workspace, ctypes.c_size_t(7), ctypes.c_size_t(7)
    assert f(1, 1, 64, 1, (1 << 26) + 1, 1, 4096, ctypes.byref(n)) == 0 and n.value == 0
    assert f(4, 2, 128, 2, 16, 8, (1 << 31) - 1, ctypes.byref(n)) == 0
    assert f(4, 2, 128, 2, 16, 8, 1 << 30, ctypes.byref(m)) == 0 and n.value == m.value > 0


def test_attention_tiles(lib):  # noqa: F811
    big = dict(ca=cache(lib, head_dim=64, n_kv_heads=1 << 13), ch=chunk(lib, rows=1 << 17), heads=1 << 13)
    assert attend(lib, pg=pages(lib, B=4096), count=40, **big) == UNSUPPORTED


@pytest.mark.parametrize("shape", [(1 << 31, 1), (1, 1 << 31), ((1 << 32) + 5, 1)])
def test_binding_refuses_shapes_beyond_32_bits(shape):
    """The library would take (2^32 + 5) rows for 5."""
    x = torch.empty(shape, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="2\\^31"):
        api._rows_2d(x, "logits", (torch.bfloat16,))
