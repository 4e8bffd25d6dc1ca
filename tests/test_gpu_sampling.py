"""Sampled tokens against the definition in 64 bits: every token equal, confidences to fp32."""
import math

import numpy as np
import pytest
import torch

import seeded_inputs as si
from paper_2608_11235_amd import DecodeState, Gate, Sched, vocab_gate, vocab_gate_sampled, vocab_sample
from tests.cache_ref import sample_row
from tests.gpu_common import log_case, require_gpu

pytestmark = pytest.mark.gpu

# sums in 64 bits, one rounding to fp32 (2^-24), one more step for the 64-bit exponential
CONF_TOL = 2.0 ** -23


def bf16(x):
    return torch.as_tensor(np.asarray(x, np.float32)).to(torch.bfloat16)


def check_rows(logits, mask_id, T, u, top_k=None, top_p=None, min_p=None, rows=None):
    """Call on the GPU, compare with the definition on (some of) the rows."""
    dev = lambda a, dt: None if a is None else torch.as_tensor(np.asarray(a)).to(dt).cuda()  # noqa: E731
    x = logits if logits.is_cuda else logits.cuda()
    tok, conf = vocab_sample(x, mask_id, dev(T, torch.float32), dev(u, torch.float32),
                             top_k=dev(top_k, torch.int32), top_p=dev(top_p, torch.float32),
                             min_p=dev(min_p, torch.float32))
    tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
    host = x.double().cpu().numpy()
    f = lambda a, r, off: off if a is None else float(np.float32(a[r]))  # noqa: E731
    for r in (range(len(host)) if rows is None else rows):
        k = 0 if top_k is None else int(top_k[r])
        want, c = sample_row(host[r], mask_id, float(np.float32(T[r])), float(np.float32(u[r])), k,
                             f(top_p, r, 1.0), f(min_p, r, 0.0))
        assert tok[r] == want, (r, tok[r], want)
        assert (math.isnan(c) and math.isnan(conf[r])) or abs(conf[r] - c) <= CONF_TOL * c, (r, conf[r], c)
    return tok, conf


def settings(rng, R):
    return {"T": rng.choice([0.0, 0.1, 0.5, 0.7, 1.0, 1.5, 30.0], size=R),
            "u": np.minimum(rng.random(R, dtype=np.float32), np.float32(1 - 2.0 ** -24)),
            "top_k": rng.choice([0, 1, 2, 7, 50, 1 << 20], size=R),
            "top_p": rng.choice([0.0, 0.3, 0.9, 0.95, 1.0], size=R),
            "min_p": rng.choice([0.0, 0.0, 0.01, 0.2, 1.0, 1.5], size=R)}


@pytest.mark.parametrize("V,R", [(1, 3), (2, 9), (7, 40), (8, 40), (13, 60), (255, 60), (2047, 60),
                                 (2048, 60), (8193, 40), (32768 + 9, 24), (50257, 16), (126464, 6),
                                 (152064, 4)])
def test_tokens_equal_the_definition(V, R):
    require_gpu()
    rng = np.random.default_rng(V)
    log_case(f"sample V={V} R={R}")
    x = bf16(rng.normal(size=(R, V)) * rng.uniform(0.3, 6.0, size=(R, 1)))
    check_rows(x, -1 if V < 3 else int(rng.integers(0, V)), **settings(rng, R))


@pytest.mark.parametrize("off", [None, "top_k", "top_p", "min_p", "all"])
def test_settings_left_out(off):
    require_gpu()
    rng = np.random.default_rng(5)
    R, V = 48, 3001
    s = settings(rng, R)
    for name in ("top_k", "top_p", "min_p"):
        if off in (name, "all"):
            s[name] = None
    check_rows(bf16(rng.normal(size=(R, V)) * 2), 17, **s)


@pytest.mark.parametrize("off,ld", [(0, 1000), (1, 1003), (3, 1008), (5, 1017), (7, 1100)])
def test_strided_rows_of_any_alignment(off, ld):
    require_gpu()
    rng = np.random.default_rng(off)
    R, V = 30, 997
    buf = bf16(rng.normal(size=(R, ld)) * 3 + 50).cuda()  # what lies beside a row is larger
    buf[:, off:off + V] -= 50
    check_rows(buf[:, off:off + V], 3, **settings(rng, R))


def test_equal_logits_go_by_id():
    require_gpu()
    rng = np.random.default_rng(11)
    R, V = 64, 4099
    x = bf16(rng.integers(-3, 3, size=(R, V)) * 0.5)
    x[::4] = 0.25                                     # every logit equal
    x[1::4] = torch.where(torch.as_tensor(rng.random((R // 4, V)) < 0.5), 0.0, -0.0).to(torch.bfloat16)
    s = settings(rng, R)
    s["u"][:8] = [0.0, 1 - 2.0 ** -24, 0.5, 0.25, 0.0, 0.75, 0.999, 0.125]
    s["T"][:8] = 1.0
    check_rows(x, 9, **s)


def test_u_at_its_ends():
    require_gpu()
    rng = np.random.default_rng(12)
    R, V = 40, 5000
    s = settings(rng, R)
    s["u"] = np.where(np.arange(R) % 2 == 0, 0.0, 1 - 2.0 ** -24).astype(np.float32)
    s["T"] = np.full(R, 0.9)
    check_rows(bf16(rng.normal(size=(R, V)) * 2), -1, **s)


LOWEST = float(torch.finfo(torch.bfloat16).min)


@pytest.mark.parametrize("fill", [-math.inf, LOWEST, -1e30, -65536.0, -2.0 ** 19, -2.0 ** 18, math.nan])
@pytest.mark.parametrize("live", [0, 1, 2, 40])
def test_banned_ids(fill, live):
    """Rows of which a fill leaves few ids, or none."""
    require_gpu()
    rng = np.random.default_rng(live)
    R, V = 24, 3000
    x = np.full((R, V), fill)
    for r in range(R):
        at = rng.choice(V, size=live, replace=False)
        x[r, at] = rng.normal(size=live) * 3
    check_rows(bf16(x), int(rng.integers(0, V)), **settings(rng, R))


@pytest.mark.parametrize("kind", ["huge", "inf", "nan", "tiny", "mask_holds_max", "mask_is_odd", "wide", "denormal"])
def test_numbers_beyond_the_common_range(kind):
    require_gpu()
    rng = np.random.default_rng(len(kind))
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
    check_rows(bf16(x), mask, **s)


@pytest.mark.parametrize("T", [-1.0, math.nan, 1e-38, 1e-4, 1e4, math.inf])
def test_odd_temperatures(T):
    require_gpu()
    rng = np.random.default_rng(3)
    R, V = 16, 1500
    s = settings(rng, R)
    s["T"] = np.full(R, T)
    check_rows(bf16(rng.normal(size=(R, V)) * 2), 0, **s)


def test_greedy_rows_equal_vocab_gate():
    require_gpu()
    R, V, mask = 32, 20011, 20000
    rng = np.random.default_rng(8)
    logits = bf16(rng.normal(size=(1, R, V))).cuda()
    prompt = si.prompt_tokens(1, 1, 8, V, mask)
    host = si.initial_decode_state(prompt, R, mask)
    a, b = (DecodeState.from_host(host, 8, R, R, R) for _ in range(2))
    zero = torch.zeros(R, device="cuda")
    vocab_gate(logits, R, -1, V, mask, a, -1, Sched(R, R), Gate(0.0, 0, True))
    vocab_gate_sampled(logits, R, -1, V, mask, b, -1, Sched(R, R), Gate(0.0, 0, True), zero, zero)
    x, y = a.to_host(), b.to_host()
    for name in x:
        if name == "conf":
            # vocab_gate sums in fp32: 2e-5 (its own tests' bound)
            assert np.allclose(x[name], y[name], rtol=2e-5, atol=0)
        else:
            assert (x[name] == y[name]).all(), name


@pytest.mark.parametrize("scope", [0, 1])
def test_gate_rules_on_sampled_tokens(scope):
    """The rules applied on the host to vocab_sample's own tokens and confidences."""
    require_gpu()
    rng = np.random.default_rng(20 + scope)
    B, P, G, blk, V, mask = 3, 10, 32, 16, 777, 700
    L = P + G
    prompt = si.prompt_tokens(1, B, P, V, mask)
    st = DecodeState.from_host(si.initial_decode_state(prompt, G, mask), P, G, G if scope else blk, blk)
    n_rows, begin = (G, P) if scope else (blk, -1)
    for step in range(6):
        before = st.to_host()
        logits = bf16(rng.normal(size=(B, n_rows, V)) * 5).cuda()
        R = B * n_rows
        T = torch.full((R,), 0.6, device="cuda")
        u = torch.as_tensor(rng.random(R, dtype=np.float32)).cuda()
        top_p = torch.full((R,), 0.9, device="cuda")
        tok, conf = vocab_sample(logits.view(R, V), mask, T, u, top_p=top_p)
        vocab_gate_sampled(logits, n_rows, begin, V, mask, st, 2, Sched(blk, 8), Gate(0.5, 1, True, scope),
                           T, u, top_p=top_p)
        after = st.to_host()
        tok, conf = tok.cpu().numpy().reshape(B, n_rows), conf.cpu().numpy().reshape(B, n_rows)
        assert (after["top1"] == tok).all() and (after["conf"] == conf).all()
        for b in range(B):
            if before["block_idx"][b] >= G // blk:
                assert (after["tokens"][b] == before["tokens"][b]).all()
                continue
            lo = P + before["block_idx"][b] * blk
            row0 = P if scope else lo
            U = before["unresolved"][b].astype(bool)
            prev, m = before["prev_top1"][b].copy(), before["persist"][b].copy()
            if not scope and before["step_idx"][b] == 0:
                prev[lo:lo + blk], m[lo:lo + blk] = -1, 0
            for p in range(row0, row0 + n_rows):
                if U[p]:
                    t = tok[b, p - row0]
                    m[p] = m[p] + 1 if prev[p] != -1 and prev[p] == t else 0
                    prev[p] = t
            cand = [p for p in range(lo, lo + blk) if U[p]]
            cand.sort(key=lambda p: (-conf[b, p - row0], p))
            commit = set(cand[:2]) | {p for p in cand[2:] if conf[b, p - row0] >= np.float32(0.5) and m[p] >= 1}
            for p in range(L):
                if p in commit:
                    assert after["tokens"][b, p] == tok[b, p - row0] and not after["unresolved"][b, p]
                else:
                    assert after["tokens"][b, p] == before["tokens"][b, p]
                    assert after["unresolved"][b, p] == before["unresolved"][b, p]
            assert (after["prev_top1"][b] == prev).all() and (after["persist"][b] == m).all()


def test_streams_graph_and_repeats():
    require_gpu()
    rng = np.random.default_rng(30)
    R, V = 40, 12345
    x = bf16(rng.normal(size=(R, V)) * 2).cuda()
    T = torch.full((R,), 0.8, device="cuda")
    u = torch.as_tensor(rng.random(R, dtype=np.float32)).cuda()
    want, wc = vocab_sample(x, 5, T, u)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [vocab_sample(x, 5, T, u, stream=s) for s in (s1, s2)]  # two calls at once
    torch.cuda.synchronize()
    tok, conf = torch.zeros_like(want), torch.zeros_like(wc)
    vocab_sample(x, 5, T, u, token=tok, conf=conf)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        vocab_sample(x, 5, T, u, token=tok, conf=conf)
    for rep in range(4):
        u.copy_(torch.as_tensor(rng.random(R, dtype=np.float32)).cuda())
        tok.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        e, ec = vocab_sample(x, 5, T, u)
        assert torch.equal(tok, e) and torch.equal(conf, ec), rep
    for t, c in outs:
        assert torch.equal(t, want) and torch.equal(c, wc)


def test_frequencies_follow_the_kept_probabilities():
    """Evenly spaced u: a token's share of them is its probability to within one draw."""
    require_gpu()
    rng = np.random.default_rng(40)
    n, V = 2048, 300
    row = bf16(rng.normal(size=V) * 2)
    x = row[None].expand(n, V).contiguous().cuda()
    u = ((torch.arange(n, dtype=torch.float32) + 0.5) / n).cuda()
    tok, _ = vocab_sample(x, -1, torch.ones(n, device="cuda"), u, top_k=torch.full((n,), 20, dtype=torch.int32, device="cuda"))
    share = np.bincount(tok.cpu().numpy(), minlength=V) / n
    l = row.double().numpy()
    order = np.argsort(-l, kind="stable")[:20]
    p = np.zeros(V)
    p[order] = np.exp(l[order]) / np.exp(l[order]).sum()
    assert np.abs(share - p).max() <= 1.0 / n + 1e-12


def test_refusals():
    require_gpu()
    x = torch.zeros((4, 10), dtype=torch.bfloat16, device="cuda")
    one = torch.ones(4, device="cuda")
    ok = dict(temperature=one, u=one * 0.5)
    from paper_2608_11235_amd._lib import CoraError
    with pytest.raises(CoraError):
        vocab_sample(x, 10, **ok)
    with pytest.raises(CoraError):
        vocab_sample(x, -2, **ok)
    with pytest.raises(ValueError, match="temperature"):
        vocab_sample(x, 0, torch.ones(3, device="cuda"), one)
    with pytest.raises(TypeError, match="top_k"):
        vocab_sample(x, 0, one, one, top_k=one)
    with pytest.raises(ValueError, match="u"):
        vocab_sample(x, 0, one, one.cpu())
    with pytest.raises(TypeError, match="logits"):
        vocab_sample(x.float(), 0, one, one)
    with pytest.raises(ValueError, match="strides"):
        vocab_sample(x.t(), 0, torch.ones(10, device="cuda"), torch.ones(10, device="cuda"))
    tok, conf = vocab_sample(x[:0], 0, one[:0], one[:0])
    assert tok.numel() == 0 and conf.numel() == 0
