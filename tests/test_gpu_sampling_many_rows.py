"""vocab_sample with more than 256 rows a call, whose kernel holds two 16-bit counts to a word:
against the definition in 64 bits, and against the same rows in smaller calls."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_common import log_case, require_gpu
from tests.test_gpu_sampling import bf16, check_rows

pytestmark = pytest.mark.gpu


def check_many(x, mask_id, s, R=300):
    """The rows of x over and over up to R rows (more than 256): the first of each against the
    definition, the others equal to it."""
    n = len(x)
    at = np.arange(R) % n
    big = x.cuda()[torch.as_tensor(at).cuda()]
    tok, conf = check_rows(big, mask_id, **{k: None if v is None else np.asarray(v)[at] for k, v in s.items()},
                           rows=range(n))
    assert (tok == tok[:n][at]).all()
    assert np.array_equal(conf, conf[:n][at], equal_nan=True)
    return tok[:n], conf[:n]


@pytest.mark.parametrize("mask", [-1, 7])
@pytest.mark.parametrize("V", [65535, 65536, 65537, 65538, 131072, 131073])
def test_more_equal_logits_than_16_bits_count(V, mask):
    """Rows of n equal logits and nothing else: 65536 of them are 0 in 16 bits."""
    require_gpu()
    counts = [n for n in (65535, 65536, 65537, 131072, V) if n <= V]
    rows = [(n, v) for n in counts for v in (-0.75, 0.75, 0.0)]
    log_case(f"equal V={V} mask={mask} counts={counts}")
    x = np.full((len(rows), V), -math.inf, np.float32)
    for r, (n, v) in enumerate(rows):
        x[r, V - n:] = v                              # the mask id among them where n is near V
    R = len(rows)
    s = {"T": np.where(np.arange(R) % 4 == 3, 0.0, 0.8), "u": (np.arange(R) * 0.37 + 0.2) % 1.0,
         "top_p": np.where(np.arange(R) % 3 == 1, 0.9, 1.0)}
    tok, _ = check_many(bf16(x), mask, s, 260)
    assert (tok >= 0).all()
    check_rows(bf16(x), mask, **s)
