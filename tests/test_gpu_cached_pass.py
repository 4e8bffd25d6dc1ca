"""The dense pass over chunks against the paged cache: logits against the oracle's layers under the
mask that the chunks amount to, and a whole sampled block decode made of the operators."""
import numpy as np
import pytest
import torch

import seeded_inputs as si
from oracle import forward as of
from paper_2608_11235_amd import (Chunk, DecodeState, Gate, KVCache, Model, Sched, cache_plan,
                                  vocab_gate_sampled, vocab_sample)
from paper_2608_11235_amd._lib import CoraError
from tests.gpu_common import log_case, require_gpu

pytestmark = pytest.mark.gpu

HD128 = si.ModelSpec("cached-hd128", 2, 256, 6, 2, 128, 512, 777, 5, True, 1e-6, 1e6, 6.0)
MODELS = {"tiny": si.TINY, "hd128": HD128}


def masked_logits(w, spec, tokens, seen):
    """Logits [L, V] of one sequence whose position i attends to the positions j with seen[i, j]."""
    L, H, Hkv, hd = len(tokens), spec.n_heads, spec.n_kv_heads, spec.head_dim
    cos, sin = of.rope_tables(L, hd, spec.rope_theta)
    h = np.asarray(w.embed_rows(tokens), np.float64)
    for i in range(spec.n_layers):
        p = {k: np.asarray(v, np.float64) for k, v in w.layer(i).items() if v is not None}
        a = of.rmsnorm(h, p["attn_norm"], spec.rms_eps)
        q, k, v = a @ p["wq"].T, a @ p["wk"].T, a @ p["wv"].T
        if spec.qkv_bias:
            q, k, v = q + p["bq"], k + p["bk"], v + p["bv"]
        q = of.rope(q.reshape(L, H, hd).transpose(1, 0, 2), cos, sin)
        k = of.rope(k.reshape(L, Hkv, hd).transpose(1, 0, 2), cos, sin)
        v = v.reshape(L, Hkv, hd).transpose(1, 0, 2)
        o = np.empty((L, H, hd))
        for j in range(H):
            s = q[j] @ k[j * Hkv // H].T / np.sqrt(hd)
            o[:, j] = of.softmax(np.where(seen, s, -np.inf)) @ v[j * Hkv // H]
        h = h + o.reshape(L, H * hd) @ p["wo"].T
        a = of.rmsnorm(h, p["mlp_norm"], spec.rms_eps)
        h = h + (of.silu(a @ p["wg"].T) * (a @ p["wu"].T)) @ p["wd"].T
    return of.logits_from_hidden(w, spec, h)


def close(got_bits, want, what):
    """Within 2e-2 of the largest logit, the bound that the dense pass's logits are held to."""
    got = got_bits.view(torch.bfloat16).double().cpu().numpy()
    err, scale = np.abs(got - want).max(), np.abs(want).max()
    log_case(f"{what}: err {err:.4f} = {err / scale:.4f} of max|l|")
    assert err <= 2e-2 * scale


def put(t, a):
    t.copy_(torch.as_tensor(np.asarray(a)).to(t.dtype))


def cache_for(spec, batch, max_len, page=32, spare=2):
    per = -(-max_len // page)
    return KVCache(spec.n_layers, batch * per + spare, spec.n_kv_heads, spec.head_dim, page, batch, per)


@pytest.mark.parametrize("name", MODELS)
@pytest.mark.parametrize("causal", [False, True])
def test_whole_sequences_in_one_chunk(name, causal):
    require_gpu()
    spec = MODELS[name]
    lens, rows = [70, 1, 33], 120
    rng = np.random.default_rng(1)
    cache, chunk = cache_for(spec, 3, 96), Chunk(3, rows)
    put(chunk.count, lens)
    cache_plan(cache, chunk)
    tokens = rng.integers(0, spec.vocab, size=rows)
    with Model(spec, 0, 2, 64) as m:
        tok = torch.as_tensor(tokens.astype(np.int32)).cuda()
        with pytest.raises(CoraError, match="128|workspace"):
            m.forward_cached(cache, Chunk(3, 129), torch.zeros(129, dtype=torch.int32, device="cuda"))
        with pytest.raises(CoraError, match="head_dim"):
            m.forward_cached(KVCache(spec.n_layers, 3, spec.n_kv_heads + 1, spec.head_dim, 32, 3, 1), chunk, tok)
    with Model(spec, 0, 2, 96) as m:
        out = m.forward_cached(cache, chunk, tok, causal=causal)
    w, at = si.HostWeights(spec, 0), 0
    for b, n in enumerate(lens):
        seen = np.tril(np.ones((n, n), bool)) if causal else np.ones((n, n), bool)
        want = masked_logits(w, spec, tokens[at:at + n], seen)
        close(out[at:at + n], want, f"{name} causal={causal} request {b}")
        if not causal:
            assert np.allclose(want, of.forward_logits(w, spec, tokens[None, at:at + n], np.arange(n))[0])
        at += n


@pytest.mark.parametrize("name", MODELS)
def test_blocks_after_a_prompt(name):
    """Prompts of different lengths in one pass, then blocks that see what is cached and, both ways,
    themselves; a block is stored anew by a second pass over it."""
    require_gpu()
    spec = MODELS[name]
    prompts, blk, n_blocks, rows = [37, 50], 16, 3, 90
    rng = np.random.default_rng(2)
    total = [p + blk * n_blocks for p in prompts]
    canvas = [rng.integers(0, spec.vocab, size=n) for n in total]
    seen = []
    for p, n in zip(prompts, total):
        group = np.maximum(0, (np.arange(n) - p) // blk + 1)
        seen.append(group[:, None] >= group[None, :])
    w = si.HostWeights(spec, 0)
    want = [masked_logits(w, spec, c, s) for c, s in zip(canvas, seen)]
    cache, chunk, block = cache_for(spec, 2, 128), Chunk(2, rows), Chunk(2, 2 * blk)
    with Model(spec, 0, 2, 128) as m:
        put(chunk.count, prompts)
        cache_plan(cache, chunk)
        tok = np.zeros(rows, np.int32)
        tok[:sum(prompts)] = np.concatenate([c[:p] for c, p in zip(canvas, prompts)])
        out = m.forward_cached(cache, chunk, torch.as_tensor(tok).cuda())
        at = 0
        for b, p in enumerate(prompts):
            close(out[at:at + p], want[b][:p], f"{name} prompt {b}")
            at += p
        for i in range(n_blocks):
            lo = [p + i * blk for p in prompts]
            put(block.start, lo)
            put(block.count, [blk, blk])
            for draft in (True, False):
                toks = np.concatenate([c[l:l + blk] for c, l in zip(canvas, lo)]).astype(np.int32)
                if draft:
                    toks[::2] = 3
                cache_plan(cache, block)
                out = m.forward_cached(cache, block, torch.as_tensor(toks).cuda(), max_count=blk, max_len=128)
            for b in range(2):
                close(out[b * blk:(b + 1) * blk], want[b][lo[b]:lo[b] + blk], f"{name} block {i} request {b}")
    assert cache.len.cpu().tolist() == total


def test_single_tokens_one_after_another():
    require_gpu()
    spec, n = HD128, 40
    rng = np.random.default_rng(3)
    tokens = rng.integers(0, spec.vocab, size=(3, n))
    w = si.HostWeights(spec, 0)
    want = [masked_logits(w, spec, t, np.tril(np.ones((n, n), bool))) for t in tokens]
    cache, chunk = cache_for(spec, 3, 64), Chunk(3, 4)
    with Model(spec, 0, 1, 64) as m:
        for i in range(n):
            put(chunk.start, [i] * 3)
            put(chunk.count, [1] * 3)
            cache_plan(cache, chunk)
            tok = torch.as_tensor(np.append(tokens[:, i], 0).astype(np.int32)).cuda()
            out = m.forward_cached(cache, chunk, tok, max_count=1, max_len=64, causal=True)
            for b in range(3):
                got = out[b].view(torch.bfloat16).double().cpu().numpy()
                assert np.abs(got - want[b][i]).max() <= 2e-2 * np.abs(want[b]).max()


def test_a_rows_logits_do_not_depend_on_its_batch():
    require_gpu()
    spec = HD128
    rng = np.random.default_rng(4)
    tok = torch.as_tensor(rng.integers(0, spec.vocab, size=96).astype(np.int32)).cuda()
    outs = []
    with Model(spec, 0, 2, 64) as m:
        for counts in ([40, 30, 7], [40, 0, 0], [40, 56, 0]):
            cache, chunk = cache_for(spec, 3, 64), Chunk(3, 96)
            put(chunk.count, counts)
            cache_plan(cache, chunk)
            outs.append(m.forward_cached(cache, chunk, tok, max_count=64, max_len=64)[:40].clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def decode(m, spec, prompt, blk, n_blocks, seed, graph):
    """Blocks decoded against the cache with sampled tokens: each step plans the active block,
    runs it, draws and applies the rules; once a block is resolved a last pass stores its tokens."""
    B, P = prompt.shape
    G = blk * n_blocks
    rng = np.random.default_rng(seed)
    u_all = torch.as_tensor(rng.random((n_blocks * (blk + 1), B * blk), dtype=np.float32)).cuda()
    cache, chunk = cache_for(spec, B, P + G), Chunk(B, B * blk)
    first = Chunk(B, B * P)
    put(first.count, [P] * B)
    cache_plan(cache, first)
    m.forward_cached(cache, first, prompt.reshape(-1), max_count=P, max_len=P + G)
    st = DecodeState.from_host(si.initial_decode_state(prompt.cpu().numpy(), G, spec.mask_id), P, G, blk, blk)
    put(chunk.count, [blk] * B)
    tok = torch.zeros(B * blk, dtype=torch.int32, device="cuda")
    u = torch.zeros(B * blk, device="cuda")
    T, top_p = torch.full((B * blk,), 0.8, device="cuda"), torch.full((B * blk,), 0.9, device="cuda")
    out = torch.empty((B * blk, spec.vocab), dtype=torch.int16, device="cuda")

    def step():
        cache_plan(cache, chunk)
        m.forward_cached(cache, chunk, tok, max_count=blk, max_len=P + G, out=out)
        vocab_gate_sampled(out, blk, -1, spec.vocab, spec.mask_id, st, -1, Sched(blk, blk), Gate(0.3, 1, True),
                           T, u, top_p=top_p)

    g = None
    if graph:
        snap = {n: getattr(st, n).clone() for n in ("tokens", "unresolved", "prev_top1", "persist", "block_idx",
                                                    "step_idx", "passes")}
        put(chunk.start, [P] * B)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            step()
        for n, t in snap.items():
            getattr(st, n).copy_(t)
    n = 0
    for i in range(n_blocks):
        lo = P + i * blk
        put(chunk.start, [lo] * B)
        while True:
            tok.copy_(st.tokens[:, lo:lo + blk].reshape(-1))
            u.copy_(u_all[n])
            done = bool((st.block_idx > i).all())
            if done:  # every token of the block is final: store its K and V
                cache_plan(cache, chunk)
                m.forward_cached(cache, chunk, tok, max_count=blk, max_len=P + G, out=out)
                break
            # rows that are ahead wait for the others: their state is put back after the step
            ahead = st.block_idx > i
            keep = {k: getattr(st, k)[ahead].clone() for k in ("tokens", "unresolved", "prev_top1", "persist",
                                                               "block_idx", "step_idx", "passes")}
            if g is not None:
                g.replay()
            else:
                step()
            for k, t in keep.items():
                getattr(st, k)[ahead] = t
            n += 1
    torch.cuda.synchronize()
    return st.to_host(), cache.len.cpu().tolist()


@pytest.mark.parametrize("name", MODELS)
def test_sampled_block_decode_over_the_cache(name):
    require_gpu()
    spec = MODELS[name]
    prompt = torch.from_numpy(si.prompt_tokens(1, 2, 21, spec.vocab, spec.mask_id)).cuda()
    with Model(spec, 0, 2, 96) as m:
        a, la = decode(m, spec, prompt, 16, 3, 5, False)
        b, lb = decode(m, spec, prompt, 16, 3, 5, True)
        c, _ = decode(m, spec, prompt, 16, 3, 6, False)
    assert la == lb == [21 + 48] * 2
    assert (a["tokens"] == b["tokens"]).all() and (a["passes"] == b["passes"]).all()
    assert (a["unresolved"] == 0).all() and (a["tokens"][:, 21:] != spec.mask_id).all()
    assert (a["tokens"][:, :21] == prompt.cpu().numpy()).all()
    assert (a["passes"] >= 1).all() and (a["passes"] <= 16).all()
    assert (a["tokens"] != c["tokens"]).any()


def test_sampled_rows_of_the_models_own_logits():
    """vocab_sample on what forward_cached writes, greedy: the lowest-id maximum of the row."""
    require_gpu()
    spec = si.TINY
    cache, chunk = cache_for(spec, 1, 64), Chunk(1, 33)
    put(chunk.count, [33])
    cache_plan(cache, chunk)
    tok = torch.from_numpy(si.prompt_tokens(3, 1, 33, spec.vocab, spec.mask_id)).cuda().view(-1)
    with Model(spec, 0, 1, 64) as m:
        out = m.forward_cached(cache, chunk, tok)
    zero = torch.zeros(33, device="cuda")
    got, conf = vocab_sample(out, spec.mask_id, zero, zero)
    x = out.view(torch.bfloat16).double().cpu()
    x[:, spec.mask_id] = -np.inf
    assert torch.equal(got.cpu().long(), x.argmax(dim=1))
    want = 1.0 / torch.exp(x - x.amax(dim=1, keepdim=True)).sum(dim=1)
    assert ((conf.cpu().double() - want).abs() <= 2.0 ** -23 * want).all()
