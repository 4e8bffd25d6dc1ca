"""The beams' choice against the definition in 64 bits: ids and parents equal, scores to fp32."""
import math

import numpy as np
import pytest
import torch

from paper_2608_11235_amd import vocab_beam, vocab_beam_workspace
from tests.beam_ref import beam_step
from tests.gpu_common import log_case, require_gpu

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.as_tensor(np.asarray(x, np.float32)).to(torch.bfloat16).cuda()


def check(x, K, W, mask_id, score, done=None, done_token=-1):
    """A thread's terms are fp32: 250 sums of 2^-24 each at the most, the exponent's argument and the hardware's
    exponential 2^-22; the rest is 64-bit and the result rounds to 2^-24 of itself.  Candidates of different
    beams nearer than that in the reference would prove nothing: there are none but equal ones."""
    sc = torch.as_tensor(np.asarray(score, np.float32)).cuda()
    d = None if done is None else torch.as_tensor(np.asarray(done, np.uint8)).cuda()
    tok, par, nxt = vocab_beam(x, K, mask_id, sc, width=W, done=d, done_token=done_token)
    host = x.double().cpu().numpy()
    want = beam_step(host, K, W, mask_id, np.asarray(score, np.float32).reshape(-1), None if done is None else np.asarray(done).reshape(-1),
                     done_token)
    assert np.array_equal(tok.cpu().numpy(), want[0]), (tok, want[0])
    assert np.array_equal(par.cpu().numpy(), want[1])
    got = nxt.cpu().numpy().astype(np.float64)
    fine = np.isfinite(want[2])
    assert np.array_equal(fine, np.isfinite(got))
    size = np.abs(want[2][fine])
    assert (np.abs(got[fine] - want[2][fine]) <= 2.0 ** -20 + 2.0 ** -24 * size).all()
    return tok, par, nxt


def scores(rng, R):
    return -rng.uniform(1, 9, size=R).astype(np.float32)


@pytest.mark.parametrize("B,K,W,V", [(1, 1, 1, 1), (2, 1, 3, 2), (3, 2, 2, 7), (2, 3, 9, 8), (4, 4, 8, 13), (2, 5, 10, 255),
                                     (1, 4, 4, 2048), (9, 2, 4, 8191), (2, 3, 6, 8193), (1, 2, 64, 16384 + 5),
                                     (1, 64, 64, 700), (1, 4, 8, 50257), (300, 2, 2, 333), (2, 8, 16, 126464),
                                     (130, 8, 16, 2047), (600, 2, 3, 9001)])
def test_random_rows(B, K, W, V):
    require_gpu()
    rng = np.random.default_rng(V + B)
    log_case(f"beam B={B} K={K} W={W} V={V}")
    x = bf16(rng.normal(size=(B * K, V)) * rng.uniform(0.3, 6.0, size=(B * K, 1)))
    check(x, K, W, -1 if V < 3 else int(rng.integers(0, V)), scores(rng, B * K))


@pytest.mark.parametrize("V", [5, 100, 9000, 40000])
@pytest.mark.parametrize("value", [0.0, -3.0e38, 2.0e38, 5.0, -1e-40, 16384.0, -20000.0])
def test_equal_logits(V, value):
    """Ties go to the lower beam, then the lower id; beams alike, and one a little ahead."""
    require_gpu()
    log_case(f"equal logits {value} V={V}")
    x = bf16(np.full((6, V), value))
    check(x, 3, 5, 2, [-1.0, -1.0, -1.0, -2.0, -1.5, -2.0])
    check(x, 3, 64, 2, [-1.0, -1.0, -1.0, -2.0, -1.5, -2.0])


@pytest.mark.parametrize("V", [9000, 30000])
@pytest.mark.parametrize("W", [1, 7, 64])
def test_rows_in_order(V, W):
    """Rising rows push every id past the bound, few different values tie everywhere."""
    require_gpu()
    log_case(f"ordered rows V={V} W={W}")
    up = np.linspace(-6, 6, V)
    steps = np.floor(np.arange(V) / 700) % 5
    x = bf16(np.stack([up, up[::-1], steps, -steps, np.sort(steps), np.abs(up)]))
    for K in (1, 3):
        check(x, K, W, V // 2, [-1.0, -1.25, -1.0, -3.0, -2.0, -2.5])


def test_zeros_of_both_signs_tie():
    require_gpu()
    x = torch.zeros((2, 50), dtype=torch.bfloat16, device="cuda")
    x[:, 1::2] = -0.0
    tok, _, _ = check(x, 2, 6, 0, [-1.0, -1.0])
    assert tok[0].tolist() == [1, 2, 3, 4, 5, 6]


@pytest.mark.parametrize("V", [40, 9000])
def test_rows_that_offer_nothing(V):
    require_gpu()
    log_case(f"rows without candidates V={V}")
    rng = np.random.default_rng(V)
    l = rng.normal(size=(12, V))
    l[0, 3], l[1, 4], l[2] = np.nan, np.inf, -np.inf
    l[3] = -np.inf
    l[3, 7] = 2.0
    l[4] = -np.inf
    l[4, 5] = 1.0            # its only id is the mask's
    l[5, 5] = np.nan         # at the mask's id: no matter
    l[6, 5] = np.inf
    l[7, :] = -3.38e38
    sc = scores(rng, 12)
    sc[8], sc[9], sc[10] = -np.inf, np.inf, np.nan
    x = bf16(l)
    for K in (1, 2, 3, 4, 12):
        check(x, K, 4, 5, sc)
    check(x, 4, 64, 5, sc)
    tok, par, nxt = check(x[:3], 3, 3, 5, sc[:3])
    assert (tok == -1).all() and (par == -1).all() and (nxt == -math.inf).all()


@pytest.mark.parametrize("V", [100, 20000])
def test_finished_beams(V):
    require_gpu()
    log_case(f"finished beams V={V}")
    rng = np.random.default_rng(1)
    x = bf16(rng.normal(size=(24, V)) * 3)
    x[3] = math.nan          # a finished beam's row is not looked at
    sc = scores(rng, 24)
    sc[5] = -np.inf
    done = np.zeros(24, np.uint8)
    done[[0, 3, 5, 8, 9, 10, 11, 20]] = 1
    for K in (1, 2, 4, 8):
        check(x, K, 6, 7, sc, done, 2)
    sc[:] = -4.0
    check(x, 4, 6, 7, sc, done, 99)
    got = vocab_beam(x, 4, 7, torch.as_tensor(sc).cuda(), width=6, done=torch.as_tensor(done).cuda().bool(), done_token=99)
    assert torch.equal(got[0], vocab_beam(x, 4, 7, torch.as_tensor(sc).cuda(), width=6, done=torch.as_tensor(done).cuda(), done_token=99)[0])


@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 5), (7, 64)])
@pytest.mark.parametrize("V", [33, 8191, 16389])
def test_strided_and_unaligned_rows(offset, pad, V):
    require_gpu()
    log_case(f"strided offset {offset} pad {pad} V={V}")
    rng = np.random.default_rng(offset)
    big = bf16(rng.normal(size=(8, offset + V + pad)) * 2)
    big[:, :offset] = 90.0
    big[:, offset + V:] = 90.0
    check(big[:, offset:offset + V], 4, 5, 3, scores(rng, 8))
    check(big[::2, offset:offset + V], 2, 5, 3, scores(rng, 4))


def test_sizes_of_logits():
    """Large, small and mixed magnitudes: what fp32 would lose of a difference stays."""
    require_gpu()
    log_case("magnitudes of logits")
    rng = np.random.default_rng(4)
    base = rng.normal(size=(8, 12000))
    for scale, shift in ((1, 1000), (1, -1000), (30, 0), (300, 0), (1e4, 0), (1e30, 0), (1e-3, 0), (1e-42, 0), (4, 16380)):
        check(bf16(base * scale + shift), 4, 8, 11, scores(rng, 8))


def test_scores_far_apart():
    require_gpu()
    rng = np.random.default_rng(5)
    x = bf16(rng.normal(size=(8, 3000)))
    for sc in ([-1e30] * 8, [0.0, -1e6, -40.0, -1e-30] * 2, [5.0, 7.0, 1e4, 2.0] * 2):
        check(x, 4, 6, 0, sc)


def test_graph_streams_and_workspace():
    require_gpu()
    rng = np.random.default_rng(6)
    log_case("beam graph")
    for B, K, V in ((2, 4, 30000), (300, 2, 5000)):
        x = bf16(rng.normal(size=(B * K, V)))
        sc = torch.as_tensor(scores(rng, B * K)).cuda()
        ws = torch.empty(vocab_beam_workspace(B, K, V, K), dtype=torch.uint8, device="cuda")
        out = vocab_beam(x, K, 0, sc, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            vocab_beam(x, K, 0, sc, token=out[0], parent=out[1], next_score=out[2], workspace=ws)
        s = torch.cuda.Stream()
        for rep in range(4):
            x.copy_(bf16(rng.normal(size=(B * K, V))))
            out[0].zero_()
            g.replay()
            torch.cuda.synchronize()
            eager = vocab_beam(x, K, 0, sc)
            s.wait_stream(torch.cuda.default_stream())
            other = vocab_beam(x, K, 0, sc, stream=s)
            torch.cuda.synchronize()
            for a, b, c in zip(out, eager, other):
                assert torch.equal(a, b) and torch.equal(a, c), rep


def test_refusals():
    require_gpu()
    x, sc = torch.zeros((6, 50), dtype=torch.bfloat16, device="cuda"), torch.zeros(6, device="cuda")
    with pytest.raises(ValueError, match="multiple"):
        vocab_beam(x, 4, 0, sc)
    with pytest.raises(ValueError, match="width"):
        vocab_beam(x, 3, 0, sc, width=0)
    with pytest.raises(ValueError, match="score"):
        vocab_beam(x, 3, 0, sc[:5])
    with pytest.raises(TypeError, match="done"):
        vocab_beam(x, 3, 0, sc, done=sc)
    with pytest.raises(ValueError, match="token"):
        vocab_beam(x, 3, 0, sc, token=torch.zeros(5, dtype=torch.int32, device="cuda"))
    from paper_2608_11235_amd._lib import CoraError
    for bad in (dict(mask_id=50), dict(mask_id=-2), dict(mask_id=0, width=65),
                dict(mask_id=0, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(CoraError):
            vocab_beam(x, 3, score=sc, **bad)
    assert vocab_beam(x[:0], 3, 0, sc[:0], width=2)[0].shape == (0, 2)
