"""Cached passes of models wide enough for the QKV projection's K to be split, over requests long
enough for several key ranges: the store's sum over slabs with and without bias, the ranges in the
workspace that held the slabs, and their merge into K panels, against the oracle's layers."""
import ctypes

import numpy as np
import pytest
import torch

import seeded_inputs as si
from paper_2608_11235_amd import Chunk, Model, _lib, cache_plan
from tests.gpu_common import log_case, require_gpu
from tests.test_gemm_plan import _split_plan
from tests.test_gpu_cached_pass import cache_for, close, masked_logits, put

#             layers  d   H Hkv hd  ffn  vocab mask bias
SPECS = {
    "d2048-hd128-bias": si.ModelSpec("wide", 2, 2048, 6, 2, 128, 512, 777, 5, True, 1e-6, 1e6, 6.0),
    "d2048-hd64": si.ModelSpec("wide", 2, 2048, 8, 2, 64, 512, 777, 5, False, 1e-6, 1e4, 6.0),
    "d1024-hd128": si.ModelSpec("wide", 2, 1024, 4, 4, 128, 320, 509, 5, False, 1e-6, 1e6, 6.0),
    "d1024-hd64-bias": si.ModelSpec("wide", 2, 1024, 7, 1, 64, 320, 509, 5, True, 1e-6, 1e4, 6.0),
}
LENS, CHUNK, MOST = [1290, 33, 700], 400, 1312


class AttnPlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("tile_rows", "tiles", "splits", "chunk", "per_request", "workgroups")] + \
        [("ws_floats", ctypes.c_size_t)]


def plans(spec, B, rows, max_count, max_len, cus=256):
    """Slabs of the QKV projection and key ranges of the attention in a pass of these sizes."""
    f = _lib.load()._ZN4cora20cache_attention_planEiiiiiiiim
    f.restype, f.argtypes = AttnPlan, [ctypes.c_int] * 8 + [ctypes.c_size_t]
    width = (spec.n_heads + 2 * spec.n_kv_heads) * spec.head_dim
    return (_split_plan(rows, width, spec.d_model, 0, 0.0).splits,
            f(B, rows, spec.n_heads, spec.n_kv_heads, spec.head_dim, max_count, max_len, cus, 1 << 25))


@pytest.mark.parametrize("name", SPECS)
@pytest.mark.parametrize("count", [1, 16, 60])
def test_sizes_reach_several_slabs_and_ranges(name, count):
    slabs, attn = plans(SPECS[name], 3, 3 * count + 2, count, MOST)
    assert slabs == (8 if "2048" in name else 4) or (count == 60 and slabs > 1)
    assert attn.splits > 1 and attn.ws_floats > 0
    G = SPECS[name].n_heads // SPECS[name].n_kv_heads
    assert (attn.tile_rows > 32) == (count * G > 32)


@pytest.mark.gpu
@pytest.mark.parametrize("name", SPECS)
@pytest.mark.parametrize("count", [1, 16, 60])
@pytest.mark.parametrize("causal", [False, True])
def test_pass_over_long_requests(name, count, causal):
    require_gpu()
    spec = SPECS[name]
    log_case(f"wide pass {name} count={count} causal={causal}")
    counts = [min(count, n) for n in LENS]
    rng = np.random.default_rng(count)
    tokens = [rng.integers(0, spec.vocab, size=n) for n in LENS]
    w, want = si.HostWeights(spec, 0), []
    for t, c in zip(tokens, counts):
        n = len(t)
        group = np.arange(n) // CHUNK                  # what is stored by one pass sees itself both ways
        group[n - c:] = group.max() + 1
        seen = np.tril(np.ones((n, n), bool)) if causal else group[:, None] >= group[None, :]
        want.append(masked_logits(w, spec, t, seen))
    cache, rows = cache_for(spec, 3, MOST), 3 * count + 2
    with Model(spec, 0, 1, MOST) as m:
        prompt, last = Chunk(3, 3 * CHUNK), Chunk(3, rows)
        tok = torch.zeros(3 * CHUNK, dtype=torch.int32, device="cuda")
        for lo in range(0, max(LENS), CHUNK):
            part = [max(0, min(CHUNK, n - c - lo)) for n, c in zip(LENS, counts)]
            put(prompt.start, [min(lo, n - c) for n, c in zip(LENS, counts)])
            put(prompt.count, part)
            new = np.concatenate([t[lo:lo + c] for t, c in zip(tokens, part)])
            tok[:len(new)] = torch.as_tensor(new.astype(np.int32)).cuda()
            cache_plan(cache, prompt)
            out = m.forward_cached(cache, prompt, tok, max_count=CHUNK, max_len=MOST, causal=causal)
            at = 0
            for b, c in enumerate(part):
                if c:
                    close(out[at:at + c], want[b][lo:lo + c], f"{name} prompt {b} from {lo}")
                at += c
        cus = torch.cuda.get_device_properties(0).multi_processor_count
        slabs, attn = plans(spec, 3, rows, count, MOST, cus)
        assert slabs > 1 and attn.splits > 1
        put(last.start, [n - c for n, c in zip(LENS, counts)])
        put(last.count, counts)
        new = np.concatenate([t[len(t) - c:] for t, c in zip(tokens, counts)] + [np.zeros(rows - sum(counts), np.int64)])
        cache_plan(cache, last)
        out = m.forward_cached(cache, last, torch.as_tensor(new.astype(np.int32)).cuda(), max_count=count, max_len=MOST,
                               causal=causal)
        at = 0
        for b, c in enumerate(counts):
            close(out[at:at + c], want[b][-c:], f"{name} request {b}")
            at += c
    assert cache.len.tolist() == LENS
