"""The beam entry point refuses malformed calls on the host, before any GPU work (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_11235_amd as pkg
from tests.beam_ref import beam_step
from tests.test_cache_abi import FAKE, INVALID, UNSUPPORTED, lib  # noqa: F401


def call(L, logits=FAKE, B=2, K=3, V=50, ld=50, mask=0, score=FAKE, done=None, W=3, token=FAKE, parent=FAKE, nxt=FAKE,
         ws=FAKE, n=1 << 40):
    return L.load().cora_vocab_beam(logits, B, K, V, ld, mask, score, done, 1, W, token, parent, nxt, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), INVALID), (dict(K=0), INVALID), (dict(W=0), INVALID), (dict(V=0), INVALID), (dict(ld=49), INVALID),
    (dict(mask=50), INVALID), (dict(mask=-2), INVALID), (dict(K=65), UNSUPPORTED), (dict(W=65), UNSUPPORTED),
    (dict(V=(1 << 30) + 1, ld=1 << 31), UNSUPPORTED), (dict(B=1 << 22, K=2), UNSUPPORTED), (dict(logits=None), INVALID),
    (dict(score=None), INVALID), (dict(token=None), INVALID), (dict(parent=None), INVALID), (dict(nxt=None), INVALID),
    (dict(ws=None), INVALID), (dict(ws=FAKE + 8), INVALID), (dict(n=15), INVALID),
    (dict(B=0, logits=None, score=None, token=None, parent=None, nxt=None, ws=None, n=0), 0)])
def test_refusals(lib, kw, status):  # noqa: F811
    assert call(lib, **kw) == status


def test_workspace(lib):  # noqa: F811
    f, n = lib.load().cora_vocab_beam_workspace, ctypes.c_size_t(0)
    for B, K, V, W in ((1, 4, 126464, 8), (128, 8, 152064, 16), (1, 1, 1, 1)):
        assert f(B, K, V, W, ctypes.byref(n)) == 0 and n.value >= B * K * (16 + 8 * W)
        assert call(lib, B=B, K=K, V=V, ld=V, W=W, n=n.value - 1) == INVALID
    assert f(1, 1, 1, 1, None) == INVALID and f(1, 0, 1, 1, ctypes.byref(n)) == INVALID
    assert f(1, 65, 1, 1, ctypes.byref(n)) == UNSUPPORTED


def test_binding_refuses_host_tensors():
    x = torch.zeros((4, 8), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        pkg.vocab_beam(x, 2, 0, torch.zeros(4))
    with pytest.raises(TypeError, match="logits"):
        pkg.vocab_beam(np.zeros((4, 8)), 2, 0, torch.zeros(4))


def test_reference():
    """The reference itself: hand-worked beams."""
    l = np.log(np.array([[0.5, 0.3, 0.2], [0.6, 0.3, 0.1]]))
    tok, par, sc = beam_step(l, 2, 3, -1, [0.0, np.log(0.5)])
    assert tok.tolist() == [[0, 0, 1]] and par.tolist() == [[0, 1, 0]]      # 0.5, 0.3 = 0.3: nearly a tie
    assert np.allclose(np.exp(sc), [[0.5, 0.3, 0.3]])
    tok, par, sc = beam_step(l, 2, 2, 0, [0.0, -np.inf])                     # id 0 left out: 0.6, 0.4
    assert tok.tolist() == [[1, 2]] and par.tolist() == [[0, 0]] and np.allclose(np.exp(sc), [[0.6, 0.4]])
    tok, par, sc = beam_step(l, 2, 3, -1, [-0.1, -5.0], [1, 0], 7)           # a finished beam in front
    assert tok.tolist() == [[7, 0, 1]] and par.tolist() == [[0, 1, 1]] and abs(sc[0, 0] + 0.1) < 1e-12
    tok, par, sc = beam_step(l[:1], 1, 5, 1, [0.0])
    assert tok.tolist() == [[0, 2, -1, -1, -1]] and par.tolist() == [[0, 0, -1, -1, -1]]
