"""Beams of long rows, several tiles a range: the loop over tiles against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2608_11235_amd import vocab_beam
from tests.gpu_common import log_case, require_gpu

pytestmark = pytest.mark.gpu

# What a row's log sum may be off by, up to 608 terms a thread (152064 ids, one range).  The exponents of the terms that are 2^8
# to 2^-8 of the thread's reference round by 2^-22 at the most and move the term by ln 2 of that, 1.65e-7; those of smaller ones,
# down to 2^-16, by twice that, but beside the largest they weigh 608 / (608 + 256) at the most: 2.4e-7 of all.  The hardware's
# exponential is off by 2^-23, a tile's 16 terms are added in four steps of 2^-24 each, and log2 e in 32 bits makes 1.3e-8
# times a distance from the reference of 5.5: 2.4 + 1.2 + 2.4 + 0.7 = 6.7e-7.
SUM = 2.0 ** -20


def reference(x, K, W, mask_id, score):
    """token, parent, score of the K W candidates of each request in order, in 64 bits."""
    R, V = x.shape
    at, cand = [], []
    for r in range(0, R, 128):
        l = x[r:r + 128].double()
        l[:, mask_id] = -math.inf
        top, order = torch.sort(l, dim=1, descending=True, stable=True)
        below = top - top[:, :1]
        cand.append(score[r:r + 128].double()[:, None] + (below[:, :W] - torch.log(torch.exp(below).sum(1, keepdim=True))))
        at.append(order[:, :W])
    row = torch.arange(R, device=x.device)[:, None].expand(R, W).reshape(R // K, K * W)
    best, order = torch.sort(torch.cat(cand).view(R // K, K * W), dim=1, descending=True, stable=True)
    return torch.gather(torch.cat(at).view(R // K, K * W), 1, order), torch.gather(row, 1, order), best


def check(x, K, W, mask_id, score, off=SUM):
    """Scores, and the order wherever no neighbour of another beam is nearer than two scores may be off."""
    token, parent, got = vocab_beam(x, K, mask_id, score, width=W)
    at, row, best = reference(x, K, W, mask_id, score)
    tol = off + 2.0 ** -24 * best[:, :W].abs()
    err = (got.double() - best[:, :W]).abs()
    log_case(f"  off by {float((err - 2.0 ** -24 * best[:, :W].abs()).max()):.2e} at the most")
    assert (err <= tol).all(), float((err - tol).max())
    near = (best[:, :-1] - best[:, 1:] <= 2 * off) & (row[:, :-1] != row[:, 1:]) & (best[:, :-1] != best[:, 1:])
    none = torch.zeros_like(near[:, :1])
    sure = ~(torch.cat([none, near], 1) | torch.cat([near, none], 1))[:, :W]
    assert sure.double().mean() > 0.99
    assert torch.equal(token.long()[sure], at[:, :W][sure])
    assert torch.equal(parent.long()[sure], row[:, :W][sure])


def normal(seed, R, V, sigma=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((R, V), dtype=torch.bfloat16, device="cuda")
    for r in range(0, R, 128):
        x[r:r + 128] = torch.randn((min(128, R - r), V), generator=g, device="cuda") * sigma
    return x


def scores(seed, R):
    return torch.as_tensor(-np.random.default_rng(seed).uniform(1, 9, size=R).astype(np.float32)).cuda()


# (requests, beams, width, ids): one range a row of 13 and 38 tiles; two, four and ten tiles a range
SIZES = [(600, 1, 4, 50257), (128, 8, 16, 152064), (8, 8, 8, 126464), (60, 4, 8, 50257), (64, 4, 64, 152064)]


@pytest.mark.parametrize("B,K,W,V", SIZES)
@pytest.mark.parametrize("height", [0, 8, 16, 30, 60])
def test_confident_ids(B, K, W, V, height):
    """An id far above the rest in the first, a middle or the last tile of a row; the mask's, in a middle tile, too."""
    require_gpu()
    log_case(f"confident ids B={B} K={K} W={W} V={V} height={height}")
    R = B * K
    x = normal(V + height, R, V)
    r = torch.arange(R, device="cuda")
    place = torch.tensor([100, V // 2 + 3, V - 3, V // 3, 5 * 4096 + 1], device="cuda")
    x[r, place[r % 5]] = float(height)
    x[r[::7], V // 2] = 50.0  # the mask's
    check(x, K, W, V // 2, scores(V, R))


@pytest.mark.parametrize("B,K,W,V", SIZES)
def test_rows_that_begin_low(B, K, W, V):
    """First tiles of nothing, of the type's lowest number, of small and of large magnitudes."""
    require_gpu()
    log_case(f"low beginnings B={B} K={K} W={W} V={V}")
    x = normal(V, B * K, V)
    x[0::5, :20000] = -math.inf
    x[1::5, :20000] = torch.finfo(torch.bfloat16).min
    x[2::5, :30000] -= 100.0
    x[3::5, :10000] -= 30000.0
    x[4::5, 30000:] -= 20000.0
    check(x, K, W, 40001, scores(V, B * K))


@pytest.mark.parametrize("B,K,W,V", SIZES)
def test_rows_in_order(B, K, W, V):
    """Rising rows push every id past the bound tile after tile, few different values tie everywhere."""
    require_gpu()
    log_case(f"ordered rows B={B} K={K} W={W} V={V}")
    up = torch.linspace(-9, 9, V, device="cuda")
    steps = torch.arange(V, device="cuda") // 700 % 5
    kinds = torch.stack([up, up.flip(0), steps, -steps, steps.sort().values, up.abs(), -up.abs(), torch.zeros_like(up)])
    x = kinds.to(torch.bfloat16).repeat(-(-B * K // 8), 1)[:B * K].contiguous()
    check(x, K, W, V // 2, scores(V + 1, B * K))


@pytest.mark.parametrize("V", [50257, 152064])
def test_equal_logits_leave_the_order_to_the_scores(V):
    """Rows of one value: its exponent, below 1/2, rounds by 2^-26, the exponential is off by 2^-23, the same for all ids, and
    sums of equal terms in powers of two are exact: 1.4e-7 a beam, so that scores 1e-6 apart keep their order."""
    require_gpu()
    log_case(f"equal logits V={V}")
    B = 300
    value = torch.tensor([3.484375, 1.4765625, 0.5, -7.71875, 12.25, -0.0203857421875], dtype=torch.bfloat16, device="cuda")
    first, second = value[torch.arange(B, device="cuda") % 6], value[torch.arange(B, device="cuda") // 6 % 6]
    x = torch.stack([first, second], 1).view(2 * B, 1).expand(2 * B, V).contiguous()
    score = torch.tensor([-1.0, -1.000001], device="cuda").repeat(B, 1)
    score[1::2] = score[1::2].flip(1)
    check(x, 2, 4, 7, score.view(-1), off=2.0 ** -22)
    token, parent, _ = vocab_beam(x, 2, 7, score.view(-1), width=4)
    ahead = torch.arange(B, device="cuda") * 2 + torch.arange(B, device="cuda") % 2
    assert (parent == ahead[:, None]).all() and (token == torch.arange(4, device="cuda")).all()


@pytest.mark.parametrize("B,V", [(4, 4096), (64, 126464), (240, 50257), (600, 50257), (1024, 152064)])
@pytest.mark.parametrize("kind", ["noise", "8", "16", "30", "60", "one value", "rising", "low first"])
def test_log_sums(B, V, kind):
    """A running score of the log sum less the largest logit leaves a best score near zero, which shows the log sum's own
    error without the score's rounding to fp32."""
    require_gpu()
    log_case(f"log sums B={B} V={V} {kind}")
    x = normal(B + V, B, V)
    g = torch.Generator(device="cuda").manual_seed(V)
    each = torch.rand((B, 1), generator=g, device="cuda")
    if kind == "one value":
        x = (each * 20 - 10).to(torch.bfloat16).expand(B, V).contiguous()
    elif kind == "rising":
        x = (torch.linspace(-9, 9, V, device="cuda") * each).to(torch.bfloat16)
    elif kind == "low first":
        x[:, :V // 3] -= 100
    elif kind != "noise":
        x[torch.arange(B, device="cuda"), torch.randint(0, V, (B,), generator=g, device="cuda")] = float(kind)
    below, top = torch.empty(B, dtype=torch.float64, device="cuda"), x.double().amax(1)
    for r in range(0, B, 128):
        below[r:r + 128] = torch.log(torch.exp(x[r:r + 128].double() - top[r:r + 128, None]).sum(1))
    score = below.float()
    got = vocab_beam(x, 1, -1, score, width=1)[2][:, 0]
    off = (got.double() - (score.double() - below)).abs()
    log_case(f"  off by {float(off.max()):.2e} at the most, {float(off.square().mean().sqrt()):.2e} rms")
    assert float(off.max()) <= 6.7e-7
