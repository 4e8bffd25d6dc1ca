"""Cached passes at positions from the model's max_seq on, which bounds the rows of a pass alone."""
import dataclasses

import numpy as np
import pytest
import torch

import seeded_inputs as si
from paper_2608_11235_amd import Chunk, KVCache, Model, cache_plan
from tests import cache_ref as ref
from tests.gpu_common import log_case, require_gpu
from tests.test_gpu_cached_pass import HD128, MODELS, cache_for, close, masked_logits, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", MODELS)
@pytest.mark.parametrize("causal", [False, True])
def test_chunks_that_pass_max_seq(name, causal):
    """Sequences of up to 200 positions in chunks of a model made for 64, then the same pass captured
    and replayed."""
    require_gpu()
    spec = MODELS[name]
    log_case(f"beyond max_seq {name} causal={causal}")
    lens, step = [200, 131], 60
    rng = np.random.default_rng(5)
    tokens = [rng.integers(0, spec.vocab, size=n) for n in lens]
    w = si.HostWeights(spec, 0)
    want = []
    for t in tokens:
        at = np.arange(len(t))
        seen = at[:, None] >= at[None, :] if causal else at[:, None] // step >= at[None, :] // step
        want.append(masked_logits(w, spec, t, seen))
    cache, chunk = cache_for(spec, 2, 224), Chunk(2, 2 * step + 3)
    with Model(spec, 0, 2, 64) as m:
        tok = torch.zeros(2 * step + 3, dtype=torch.int32, device="cuda")
        for lo in range(0, max(lens), step):
            count = [max(0, min(step, n - lo)) for n in lens]
            put(chunk.start, [min(lo, n) for n in lens])
            put(chunk.count, count)
            rows = np.concatenate([t[lo:lo + c] for t, c in zip(tokens, count)])
            tok[:len(rows)] = torch.as_tensor(rows.astype(np.int32)).cuda()
            cache_plan(cache, chunk)
            out = m.forward_cached(cache, chunk, tok, max_count=step, max_len=224, causal=causal)
            assert chunk.status.tolist() == [0, 0]
            at = 0
            for b, c in enumerate(count):
                if c:
                    close(out[at:at + c], want[b][lo:lo + c], f"{name} request {b} from {lo}")
                at += c
        again = torch.zeros_like(out)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            m.forward_cached(cache, chunk, tok, max_count=step, max_len=224, causal=causal, out=again)
        for _ in range(3):
            again.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(again[:len(rows)], out[:len(rows)])


def test_positions_of_the_table_keep_their_angles():
    """A cache with room beyond the table of angles: what the table has is stored bit for bit as
    with a cache without."""
    require_gpu()
    spec = HD128
    rng = np.random.default_rng(6)
    tok = torch.as_tensor(rng.integers(0, spec.vocab, size=60).astype(np.int32)).cuda()
    outs, keys = [], []
    with Model(spec, 0, 1, 64) as m:
        for room in (64, 96):
            cache, chunk = cache_for(spec, 1, room), Chunk(1, 60)
            put(chunk.count, [60])
            cache_plan(cache, chunk)
            outs.append(m.forward_cached(cache, chunk, tok, max_count=60, max_len=64).clone())
            keys.append(cache.k[:, :2].clone())
    assert torch.equal(outs[0], outs[1])
    ko = ref.offsets(32, spec.head_dim)[0]
    a, b = (ref.natural(k, ko).transpose(1, 2).reshape(spec.n_layers, spec.n_kv_heads, 64, -1)[:, :, :60] for k in keys)
    assert torch.equal(a, b)


@pytest.mark.parametrize("far", [64, 1000, 70001, (1 << 29) + 12345])
@pytest.mark.parametrize("hd", [64, 128])
def test_far_positions(hd, far):
    """The keys of a token at position 3 and far out: the same ones, turned by the angle between."""
    require_gpu()
    log_case(f"far position {far} hd={hd}")
    spec = dataclasses.replace(HD128, n_layers=1, head_dim=hd, n_heads=256 // hd, n_kv_heads=1)
    page = 256
    pages = -(-(far + 1) // page)
    cache, chunk = KVCache(1, 4, 1, hd, page, 1, pages), Chunk(1, 1)
    cache.table.fill_(1)
    ko = ref.offsets(page, hd)[0]
    k = []
    with Model(spec, 0, 1, 8) as m:
        for pos in (3, far):
            put(cache.len, [1])                        # what the row attends to is not looked at
            put(chunk.cu, [0, 1]); put(chunk.start, [pos]); put(chunk.positions, [pos])
            put(chunk.slots, [2 * page + pos % page])
            tok = torch.full((1,), 17, dtype=torch.int32, device="cuda")
            cache.k.zero_(); cache.v.zero_()
            m.forward_cached(cache, chunk, tok, max_count=1, max_len=256)
            k.append(ref.natural(cache.k[0], ko)[2, 0, pos % page].double().cpu().numpy())
    ang = (far - 3) * spec.rope_theta ** (-2.0 * np.arange(hd // 2) / hd)
    a, b = k[0][0::2], k[0][1::2]
    c, s = np.cos(ang), np.sin(ang)
    want = np.stack([a * c - b * s, b * c + a * s], -1).reshape(-1)
    # both keys are rounded to bf16 (2^-8 of what they hold), their angles' cos and sin to fp32
    # (2^-24), and the angle's product in 64 bits is off by 2^-53 of it, which is below 2^30
    mag = np.stack([abs(a * c) + abs(b * s), abs(b * c) + abs(a * s)], -1).reshape(-1)
    size = np.repeat(np.hypot(a, b), 2)
    tol = 2.0 ** -8 * (abs(want) + mag) * (1 + 2.0 ** -7) + size * (4 * 2.0 ** -24 + 2 * 2.0 ** -23)
    assert np.abs(k[0]).max() > 0 and (np.abs(k[1] - want) <= tol).all(), float((np.abs(k[1] - want) / tol).max())
