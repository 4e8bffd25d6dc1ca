"""vocab_sample with more than 256 rows a call, whose kernel holds two 16-bit counts to a word:
against the definition in 64 bits, and against the same rows in smaller calls."""
import math

import numpy as np
import pytest
import torch

import seeded_inputs as si
from paper_2608_11235_amd import DecodeState, Gate, Sched, vocab_gate_sampled, vocab_sample
from tests.gpu_common import log_case, require_gpu
from tests.test_gpu_sampling import LOWEST, bf16, check_rows, settings

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


@pytest.mark.parametrize("V,n", [(1, 3), (2, 9), (7, 40), (8, 40), (13, 60), (255, 60), (2047, 60), (2048, 60),
                                 (8193, 40), (32768 + 9, 24), (50257, 12), (126464, 5), (152064, 3)])
def test_tokens_equal_the_definition(V, n):
    require_gpu()
    rng = np.random.default_rng(V + 1)
    log_case(f"sample many V={V}")
    x = bf16(rng.normal(size=(n, V)) * rng.uniform(0.3, 6.0, size=(n, 1)))
    check_many(x, -1 if V < 3 else int(rng.integers(0, V)), settings(rng, n), 257 if V > 1 << 16 else 600)


@pytest.mark.parametrize("off,ld", [(0, 1000), (1, 1003), (3, 1008), (5, 1017), (7, 1100)])
def test_strided_rows_of_any_alignment(off, ld):
    require_gpu()
    rng = np.random.default_rng(off + 50)
    R, V = 290, 997
    buf = bf16(rng.normal(size=(R, ld)) * 3 + 50).cuda()  # what lies beside a row is larger
    buf[:, off:off + V] -= 50
    check_rows(buf[:, off:off + V], 3, **settings(rng, R), rows=range(0, R, 7))


@pytest.mark.parametrize("mask", [-1, 9])
def test_equal_logits_go_by_id(mask):
    require_gpu()
    rng = np.random.default_rng(51)
    R, V = 64, 4099
    x = bf16(rng.integers(-3, 3, size=(R, V)) * 0.5)
    x[::4] = 0.25
    x[1::4] = torch.where(torch.as_tensor(rng.random((R // 4, V)) < 0.5), 0.0, -0.0).to(torch.bfloat16)
    x[2::8] = -0.25
    s = settings(rng, R)
    s["u"][:8] = [0.0, 1 - 2.0 ** -24, 0.5, 0.25, 0.0, 0.75, 0.999, 0.125]
    s["T"][:8] = 1.0
    check_many(x, mask, s)


@pytest.mark.parametrize("value", [-2.0, -0.0, 0.0, 2.0])
def test_the_mask_ids_count_in_either_half(value):
    """The mask id alone holds its number, or the number's negative has many ids in the same word."""
    require_gpu()
    rng = np.random.default_rng(52)
    R, V, mask = 32, 1200, 600
    x = rng.normal(size=(R, V))
    x[8:16] = -value
    x[16:24] = -abs(rng.normal(size=(8, V))) - 3
    x[24:] = value
    x[:, mask] = value
    check_many(bf16(x), mask, settings(rng, R))


@pytest.mark.parametrize("fill", [-math.inf, LOWEST, -1e30, -65536.0, -2.0 ** 19, -2.0 ** 18, math.nan])
@pytest.mark.parametrize("live", [0, 1, 2, 40])
def test_banned_ids(fill, live):
    require_gpu()
    rng = np.random.default_rng(live + 60)
    R, V = 24, 3000
    x = np.full((R, V), fill)
    for r in range(R):
        at = rng.choice(V, size=live, replace=False)
        x[r, at] = rng.normal(size=live) * 3
    check_many(bf16(x), int(rng.integers(0, V)), settings(rng, R))


@pytest.mark.parametrize("kind", ["huge", "inf", "nan", "tiny", "mask_holds_max", "mask_is_odd", "wide", "denormal"])
def test_numbers_beyond_the_common_range(kind):
    require_gpu()
    rng = np.random.default_rng(len(kind) + 70)
    R, V, mask = 32, 2500, 77
    x = rng.normal(size=(R, V)) * 2
    if kind == "huge":
        x[:, ::7] *= 1e6
    elif kind == "inf":
        x[::2, 5] = math.inf
        x[::3, 9] = math.inf
    elif kind == "nan":
        x[::2, 5] = math.nan
        x[1, :] = math.nan
    elif kind == "tiny":
        x *= 2.0 ** -46
    elif kind == "mask_holds_max":
        x[:, mask] = 100.0
        x[::2, mask] = 1e30
    elif kind == "mask_is_odd":
        x[:, mask] = np.where(np.arange(R) % 3 == 0, math.nan, np.where(np.arange(R) % 3 == 1, math.inf, LOWEST))
    elif kind == "wide":
        x = np.exp(rng.uniform(-60, 60, size=(R, V))) * rng.choice([-1, 1], size=(R, V))
    elif kind == "denormal":
        x = x * 1e-39
    s = settings(rng, R)
    if kind in ("huge", "wide"):
        s["T"] = rng.choice([0.5, 1.0, 1e5, 1e30], size=R)
    check_many(bf16(x), mask, s)


@pytest.mark.parametrize("T", [-1.0, math.nan, 1e-38, 1e-4, 1e4, math.inf])
def test_odd_temperatures(T):
    require_gpu()
    rng = np.random.default_rng(80)
    R, V = 16, 1500
    s = settings(rng, R)
    s["T"] = np.full(R, T)
    check_many(bf16(rng.normal(size=(R, V)) * 2), 0, s)


@pytest.mark.parametrize("off", ["top_k", "top_p", "min_p", "all"])
def test_settings_left_out(off):
    require_gpu()
    rng = np.random.default_rng(90)
    R, V = 48, 3001
    s = settings(rng, R)
    for name in ("top_k", "top_p", "min_p"):
        if off in (name, "all"):
            s[name] = None
    check_many(bf16(rng.normal(size=(R, V)) * 2), 17, s)


@pytest.mark.parametrize("V", [500, 40009])
def test_256_and_257_rows_give_the_same(V):
    """The two kernels, which a call's number of rows chooses between, take the same sums."""
    require_gpu()
    rng = np.random.default_rng(V)
    R = 257
    x = bf16(rng.normal(size=(R, V)) * 2.5).cuda()
    s = settings(rng, R)
    dev = {k: torch.as_tensor(v).to(torch.int32 if k == "top_k" else torch.float32).cuda() for k, v in s.items()}
    call = lambda n: vocab_sample(x[:n], 11, dev["T"][:n], dev["u"][:n], top_k=dev["top_k"][:n],  # noqa: E731
                                  top_p=dev["top_p"][:n], min_p=dev["min_p"][:n])
    (a, ca), (b, cb) = call(256), call(257)
    assert torch.equal(a, b[:256]) and torch.equal(ca, cb[:256])


def test_gate_on_a_whole_generation_region():
    """The rules take these kernels' tokens and confidences too: 3 x 112 rows in GLOBAL scope."""
    require_gpu()
    rng = np.random.default_rng(95)
    B, P, G, blk, V, mask = 3, 5, 112, 16, 1009, 1000
    R = B * G
    host = si.initial_decode_state(si.prompt_tokens(1, B, P, V, mask), G, mask)
    st = DecodeState.from_host(host, P, G, G, blk)
    logits = bf16(rng.normal(size=(B, G, V)) * 4).cuda()
    T, u = torch.full((R,), 0.7, device="cuda"), torch.as_tensor(rng.random(R, dtype=np.float32)).cuda()
    tok, conf = vocab_sample(logits.view(R, V), mask, T, u)
    vocab_gate_sampled(logits, G, P, V, mask, st, 2, Sched(blk, 8), Gate(0.5, 1, True, 1), T, u)
    after = st.to_host()
    tok, conf = tok.cpu().numpy().reshape(B, G), conf.cpu().numpy().reshape(B, G)
    assert (after["top1"] == tok).all() and (after["conf"] == conf).all()
    for b in range(B):
        first = sorted(range(blk), key=lambda p: (-conf[b, p], p))[:2]  # the gate needs a repeated draw
        want = host["tokens"][b].copy()
        want[[P + p for p in first]] = tok[b, first]
        assert (after["tokens"][b] == want).all()
