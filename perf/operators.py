"""The work that the performance of the cached and sampled decode's operators is measured on.

Four operators make up a serving step that keeps K and V instead of recomputing the canvas and
that draws its tokens instead of taking the largest logit:

    plan    block tables and slot maps of a batch of requests, from their lengths
    store   rotary positions on the q and k of a chunk of new tokens; k and v into the pages
    attend  attention of the chunk over each request's pages
    sample  a token per logits row by temperature, top-k, top-p and min-p from a given random
            number, with its confidence

`run` computes them in elementary torch operations, or calls the package's operators.  Pages hold
K and V in the order of the package's matrix operands; `k_offsets` and `v_offsets` say where.
"""
import math

import numpy as np
import torch

own = False


# ---- the cases ------------------------------------------------------------------------------
def _sample(name, rows, vocab, ld, params, sigma):
    return {"name": name, "kind": "sample", "rows": rows, "vocab": vocab, "ld": ld,
            "params": params, "sigma": sigma}


def _plan(name, batch, page, most, count, reset):
    return {"name": name, "kind": "plan", "batch": batch, "page": page, "most": most,
            "count": count, "reset": reset}


def _store(name, batch, count, ragged, heads, kv_heads, head_dim, page, most):
    return {"name": name, "kind": "store", "batch": batch, "count": count, "ragged": ragged,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "most": most}


def _attend(name, batch, count, ragged, heads, kv_heads, head_dim, page, least, most, causal):
    return {"name": name, "kind": "attend", "batch": batch, "count": count, "ragged": ragged,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
            "least": least, "most": most, "causal": causal}


def listed():
    return [
        # the tiny model's vocabulary, the 16 rows of its block: latency alone
        _sample("sample_tiny", 16, 2048, 2048, "top_p", 2.5),
        # the active block of one LLaDA-8B sequence, nucleus sampling
        _sample("sample_block", 32, 126464, 126464, "top_p", 1.3),
        # a vocabulary of odd size in padded rows, every request with settings of its own
        _sample("sample_mixed_odd", 777, 50257, 50261, "mixed", 2.0),
        # whole canvases of eight sequences, the vocab/gate workload's logits: the largest
        _sample("sample_canvas", 4096, 126464, 126464, "top_p", 1.0),
        # one more token for each of 64 running requests
        _plan("plan_tokens", 64, 64, 8192, 1, False),
        # a fresh batch of 512 prompts of up to 2048 tokens: tables built from nothing
        _plan("plan_prompts", 512, 64, 2048, 0, True),
        # one new token for each of 64 requests, Dream-7B heads: latency
        _store("store_tokens", 64, 1, False, 28, 4, 128, 64, 4096),
        # the prompts and canvases of eight LLaDA-8B sequences
        _store("store_canvas", 8, 512, False, 32, 32, 128, 64, 512),
        # a block of 16 on a short canvas of the tiny model: launches and latency
        _attend("attend_tiny", 1, 16, False, 4, 4, 64, 32, 96, 96, False),
        # one token each of 64 requests over 64 to 8192 cached ones, Dream-7B heads: a stream of K, V
        _attend("attend_tokens", 64, 1, False, 28, 4, 128, 64, 64, 8192, True),
        # the active block of eight LLaDA-8B sequences over up to 1280 positions, both directions
        _attend("attend_blocks", 8, 32, False, 32, 32, 128, 64, 288, 1280, False),
        # the second half of four prompts of 4096 tokens, Dream-7B heads: matrix products
        _attend("attend_prompts", 4, 2048, False, 28, 4, 128, 128, 4096, 4096, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 to 4096 rows of 500 to 152064 logits; 1 to 512 requests, chunks of one
    token to a few thousand, up to 16384 cached ones; 64- and 128-wide heads, shared or not;
    pages of 32 to 256."""
    kind = rng.choice(["sample", "sample", "plan", "store", "attend", "attend", "attend"])
    if kind == "sample":
        vocab = _log_int(rng, 500, 152064)
        rows = _log_int(rng, 1, max(1, min(4096, 200_000_000 // vocab)))
        case = _sample("", rows, vocab, vocab + rng.choice([0, 0, 1, 3, 8, 64]),
                       rng.choice(["top_p", "mixed", "mixed"]), rng.uniform(0.7, 4.0))
    elif kind == "plan":
        count = rng.choice([0, 1, 8, 32])
        case = _plan("", _log_int(rng, 1, 512), rng.choice([32, 64, 128, 256]),
                     _log_int(rng, 64, 2048 if count == 0 else 8192), count, count == 0)
    else:
        kv_heads = rng.choice([1, 2, 4, 8, 16, 32])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
        heads = heads if heads <= 64 else kv_heads
        head_dim, page = rng.choice([64, 128]), rng.choice([32, 64, 128, 256])
        batch = _log_int(rng, 1, 64)
        if kind == "store":
            count = _log_int(rng, 1, max(1, 4096 // batch))
            case = _store("", batch, count, rng.random() < 0.5, heads, kv_heads, head_dim, page,
                          count + _log_int(rng, 1, 1024))
        else:
            # the K and V of all requests fit 512 MB, the products the largest listed case's
            most = max(64, min(16384, 2 ** 29 // (batch * kv_heads * head_dim * 4)))
            most = _log_int(rng, 48, most)
            count = _log_int(rng, 1, max(1, min(most, 4096 // batch)))
            while count > 1 and 4 * batch * count * most * heads * head_dim > 2.4e11:
                count = (count + 1) // 2
            case = _attend("", batch, count, rng.random() < 0.5, heads, kv_heads, head_dim, page,
                           max(count, most // 8), most, rng.random() < 0.5)
    del case["name"]
    return case


# ---- the order of K and V in a page -----------------------------------------------------------
def k_offsets(page, head_dim):
    """[page, head_dim]: where a page's block of one kv head holds K.  32-key groups of two
    halves, each head_dim / 32 blocks of 16 keys x 32 dimensions: lane r + 16 g of a block holds
    dimensions 8 g .. 8 g + 7 of key 8 (r / 4) + 4 half + r % 4."""
    p = torch.arange(page)[:, None]
    d = torch.arange(head_dim)[None, :]
    k = p % 32
    r = 4 * (k // 8) + k % 4
    return (p // 32) * 32 * head_dim + (k % 8 // 4) * 16 * head_dim + (d // 32) * 512 \
        + (d % 32 // 8) * 128 + r * 8 + d % 8


def v_offsets(page, head_dim):
    """[page, head_dim]: where it holds V.  32-key groups of head_dim / 16 blocks of 16
    dimensions x 32 keys: lane r + 16 g holds keys 8 g .. 8 g + 7 of dimension r."""
    p = torch.arange(page)[:, None]
    d = torch.arange(head_dim)[None, :]
    k = p % 32
    return (p // 32) * 32 * head_dim + (d // 16) * 512 + (k // 8) * 128 + (d % 16) * 8 + k % 8


# ---- inputs ---------------------------------------------------------------------------------
def _dev(x, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(x)).to(dtype).cuda() if dtype else \
        torch.as_tensor(np.ascontiguousarray(x)).cuda()


def _logits(case, gen, rng):
    """N(0, sigma) with a spike of up to 12 in most rows, as a model's own rows have; the ids of
    a banned few hold bf16's lowest number or -inf in some rows."""
    R, V, ld = case["rows"], case["vocab"], case["ld"]
    out = torch.empty((R, ld), dtype=torch.bfloat16, device="cuda")
    for r0 in range(0, R, 512):
        n = min(512, R - r0)
        x = torch.randn((n, ld), generator=gen, device="cuda") * case["sigma"]
        at = _dev(rng.integers(0, V, size=n))
        x[torch.arange(n, device="cuda"), at] += _dev(rng.uniform(0.0, 12.0, size=n).astype(np.float32))
        out[r0:r0 + n] = x
    for r in range(0, R, 16):
        out[r, 5:V // 50] = -math.inf if r % 32 else torch.finfo(torch.bfloat16).min
    return out[:, :V]


def _sample_params(case, rng):
    R = case["rows"]
    f32 = np.float32
    if case["params"] == "top_p":
        return {"temperature": np.full(R, 0.7, f32), "top_k": None, "top_p": np.full(R, 0.95, f32),
                "min_p": None}
    return {"temperature": rng.choice(np.array([0.0, 0.2, 0.6, 0.8, 1.0, 1.3], f32), size=R),
            "top_k": rng.choice(np.array([0, 1, 20, 50, 1000], np.int32), size=R),
            "top_p": rng.choice(np.array([0.5, 0.9, 0.95, 1.0], f32), size=R),
            "min_p": rng.choice(np.array([0.0, 0.0, 0.02, 0.1], f32), size=R)}


def _prepare_sample(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    logits = _logits(case, gen, rng)
    par = {k: None if v is None else _dev(v) for k, v in _sample_params(case, rng).items()}
    u = _dev(rng.random(case["rows"], dtype=np.float32))
    return {"kind": "sample", "logits": logits, "mask_id": case["vocab"] - case["vocab"] // 1000 - 1,
            "u": u, **par}


def _lengths(case, rng):
    """(start, count, cached) of each request: a chunk of `count` new tokens at the end."""
    B = case["batch"]
    if case["kind"] == "plan":
        if case["count"] == 0:
            n = rng.integers(1, case["most"] + 1, size=B)
            return np.zeros(B, np.int64), n
        start = rng.integers(1, max(2, case["most"] - case["count"] + 1), size=B)
        return start, np.full(B, case["count"])
    count = np.full(B, case["count"])
    if case["ragged"]:
        count = rng.integers(1, case["count"] + 1, size=B)
        count[rng.integers(0, B)] = case["count"]
    if case["kind"] == "store":
        return rng.integers(0, case["most"] - case["count"] + 1, size=B), count
    lo = max(case["least"], case["count"])
    total = np.exp(rng.uniform(math.log(lo), math.log(max(lo, case["most"])), size=B))
    total = np.minimum(np.round(total).astype(np.int64), max(lo, case["most"]))
    total[rng.integers(0, B)] = max(lo, case["most"])
    return total - count, count


def _requests(case, seed):
    """The batch of a plan, store or attention case on the host: chunks, cached lengths, block
    tables over pages in random order, and the stack of free ones.  The lengths are the case's;
    the seed says which request has which of them, and which pages."""
    start, count = _lengths(case, np.random.default_rng([case["batch"], case["page"], case["most"]]))
    rng = np.random.default_rng(seed)
    who = rng.permutation(case["batch"])
    start, count = start[who], count[who]
    page = case["page"]
    if case["kind"] == "plan":
        cached = np.zeros_like(start) if case["reset"] else start
    else:
        cached = start + count
    after = -(-(start + count) // page)
    have = -(-cached // page)
    max_pages = int(after.max())
    n_pages = int(after.sum()) + (7 if case["kind"] == "plan" else 0)
    order = rng.permutation(n_pages)
    table = np.full((case["batch"], max_pages), -1, np.int32)
    at = 0
    for b in range(case["batch"]):
        table[b, :have[b]] = order[at:at + have[b]]
        at += have[b]
    free = np.zeros(n_pages, np.int32)
    free[:n_pages - at] = order[at:]
    i32 = np.int32
    return rng, {"start": start.astype(i32), "count": count.astype(i32), "len": cached.astype(i32),
                 "table": table, "free": free, "n_free": np.array([n_pages - at], i32),
                 "n_pages": n_pages, "max_pages": max_pages, "page": page,
                 "cu": np.concatenate([[0], np.cumsum(count)]).astype(i32), "rows": int(count.sum())}


def _row_maps(req):
    """Position and slot of every row of the chunks."""
    pos = np.concatenate([s + np.arange(c) for s, c in zip(req["start"], req["count"])])
    b = np.repeat(np.arange(len(req["count"])), req["count"])
    slots = req["table"][b, pos // req["page"]].astype(np.int64) * req["page"] + pos % req["page"]
    return pos.astype(np.int32), slots.astype(np.int32)


def _cache_of(case, req, k, v, kv_heads, head_dim):
    from paper_2608_11235_amd import KVCache
    cache = KVCache(1, req["n_pages"], kv_heads, head_dim, req["page"], case["batch"],
                    req["max_pages"])
    if k is not None:
        cache.k[0].copy_(k)
        cache.v[0].copy_(v)
    for name in ("table", "len", "free", "n_free"):
        getattr(cache, name).copy_(_dev(req[name]))
    return cache


def _chunk_of(case, req, maps):
    from paper_2608_11235_amd import Chunk
    chunk = Chunk(case["batch"], req["rows"])
    chunk.start.copy_(_dev(req["start"]))
    chunk.count.copy_(_dev(req["count"]))
    if maps is not None:
        chunk.cu.copy_(_dev(req["cu"]))
        chunk.positions.copy_(_dev(maps[0]))
        chunk.slots.copy_(_dev(maps[1]))
    return chunk


def _prepare_plan(case, seed):
    _, req = _requests(case, seed)
    st = {"kind": "plan", "reset": case["reset"], "page": req["page"], "n_pages": req["n_pages"],
          "max_pages": req["max_pages"], "rows": req["rows"]}
    if own:
        st["cache"] = _cache_of(case, req, None, None, 1, 64)
        st["chunk"] = _chunk_of(case, req, None)
    else:
        for name in ("start", "count", "len", "table", "free", "n_free"):
            st[name] = _dev(req[name])
    return st


def _prepare_store(case, seed):
    rng, req = _requests(case, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    H, Hkv, hd = case["heads"], case["kv_heads"], case["head_dim"]
    x = torch.randn((req["rows"], (H + 2 * Hkv) * hd), generator=gen, device="cuda").to(torch.bfloat16)
    shape = (req["n_pages"], Hkv, req["page"] * hd)
    k = torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    v = torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    ang = torch.arange(case["most"], dtype=torch.float64)[:, None] \
        * 1e6 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64)[None, :] / hd)
    rope = torch.stack([torch.cos(ang), torch.sin(ang)], dim=-1).to(torch.float32).cuda()
    maps = _row_maps(req)
    st = {"kind": "store", "heads": H, "kv_heads": Hkv, "head_dim": hd, "page": req["page"], "x": x,
          "rope": rope}
    if own:
        st["cache"] = _cache_of(case, req, k, v, Hkv, hd)
        st["chunk"] = _chunk_of(case, req, maps)
        st["q"] = torch.empty((req["rows"], H, hd), dtype=torch.bfloat16, device="cuda")
    else:
        st.update(k=k, v=v, positions=_dev(maps[0]), slots=_dev(maps[1]))
    return st


def _prepare_attend(case, seed):
    rng, req = _requests(case, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    H, Hkv, hd = case["heads"], case["kv_heads"], case["head_dim"]
    q = torch.randn((req["rows"], H, hd), generator=gen, device="cuda").to(torch.bfloat16)
    shape = (req["n_pages"], Hkv, req["page"] * hd)
    k = torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    v = torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    st = {"kind": "attend", "q": q, "heads": H, "kv_heads": Hkv, "head_dim": hd, "page": req["page"],
          "causal": case["causal"], "max_count": int(req["count"].max()),
          "max_len": int(req["len"].max())}
    if own:
        st["cache"] = _cache_of(case, req, k, v, Hkv, hd)
        st["chunk"] = _chunk_of(case, req, _row_maps(req))
        st["out"] = torch.empty_like(q)
    else:
        st.update(k=k, v=v, table=_dev(req["table"]).long(), starts=req["start"].tolist(),
                  counts=req["count"].tolist(), lens=req["len"].tolist())
    return st


def prepare(case, seed):
    return {"sample": _prepare_sample, "plan": _prepare_plan, "store": _prepare_store,
            "attend": _prepare_attend}[case["kind"]](case, seed)


# ---- one pass ---------------------------------------------------------------------------------
def _plain_sample(st):
    """Sorted by logit (ties by id), the kept ones a prefix; sums in 64 bits, since a token is
    decided where a running sum of up to 152064 terms passes a number."""
    logits, mask_id = st["logits"], st["mask_id"]
    R, V = logits.shape
    tokens, confs = [], []
    step = max(1, 16_000_000 // V)
    for r0 in range(0, R, step):
        sl = slice(r0, min(R, r0 + step))
        x = logits[sl].float().clone()
        x[:, mask_id] = -math.inf
        val, idx = torch.sort(x, dim=1, descending=True, stable=True)
        below = (val - val[:, :1]).double()
        T = st["temperature"][sl].double()[:, None]
        w = torch.exp(below / torch.where(T > 0, T, torch.ones_like(T)))
        w = torch.where(below == -math.inf, torch.zeros_like(w), w)
        rank = torch.arange(V, device="cuda")[None, :]
        keep = torch.ones_like(val, dtype=torch.bool)
        if st["top_k"] is not None:
            k = st["top_k"][sl][:, None]
            keep &= (k <= 0) | (rank < k)
        cum = torch.cumsum(torch.where(keep, w, torch.zeros_like(w)), dim=1)
        if st["top_p"] is not None:
            p = st["top_p"][sl].double()[:, None]
            before = torch.nn.functional.pad(cum[:, :-1], (1, 0))
            keep &= (p >= 1) | (before < p * cum[:, -1:]) | (rank == 0)
        if st["min_p"] is not None:
            m = st["min_p"][sl].double()[:, None]
            keep &= (m <= 0) | (w >= m) | (rank == 0)
        last = keep.sum(dim=1, keepdim=True) - 1
        target = st["u"][sl].double()[:, None] * torch.gather(cum, 1, last)
        j = torch.minimum((cum <= target).sum(dim=1, keepdim=True), last)
        j = torch.where(T > 0, j, torch.zeros_like(j))
        e = torch.exp(below)
        tokens.append(torch.gather(idx, 1, j)[:, 0].to(torch.int32))
        confs.append((torch.gather(e, 1, j)[:, 0] / e.sum(dim=1)).float())
    return {"token": torch.cat(tokens), "conf": torch.cat(confs)}


def _plain_plan(st):
    """Prefix sums over the requests, then every page and every row looks its request up."""
    page, n_pages, rows = st["page"], st["n_pages"], st["rows"]
    start, count = st["start"].long(), st["count"].long()
    if st["reset"]:
        st["len"].zero_()
        st["free"].copy_(torch.arange(n_pages - 1, -1, -1, device="cuda"))
        st["n_free"].fill_(n_pages)
    have = (st["len"].long() + page - 1) // page
    length = torch.maximum(st["len"].long(), start + count)
    need = (length + page - 1) // page - have
    first = torch.cumsum(need, 0) - need
    B, max_pages = st["table"].shape
    j = torch.arange(max_pages, device="cuda")[None, :]
    new = (j >= have[:, None]) & (j < (have + need)[:, None])
    at = st["n_free"].long() - 1 - (first[:, None] + j - have[:, None])
    taken = st["free"][at.clamp(0, n_pages - 1)]
    st["table"].copy_(torch.where(new, taken, st["table"]))
    st["n_free"].sub_(need.sum().to(torch.int32))
    st["len"].copy_(length)
    cu = torch.zeros(B + 1, dtype=torch.int64, device="cuda")
    cu[1:] = torch.cumsum(count, 0)
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(cu, r, right=True) - 1
    pos = start[b] + r - cu[b]
    slots = st["table"][b, pos // page].long() * page + pos % page
    i32 = torch.int32
    return {"cu": cu.to(i32), "positions": pos.to(i32), "slots": slots.to(i32),
            "status": torch.zeros(B, dtype=i32, device="cuda"), "table": st["table"],
            "len": st["len"], "free": st["free"], "n_free": st["n_free"]}


def _rotate(x, cs):
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _plain_store(st):
    H, Hkv, hd, page = st["heads"], st["kv_heads"], st["head_dim"], st["page"]
    x = st["x"].float().view(-1, H + 2 * Hkv, hd)
    cs = st["rope"][st["positions"].long()]
    q, k = _rotate(x[:, :H], cs).to(torch.bfloat16), _rotate(x[:, H:H + Hkv], cs).to(torch.bfloat16)
    v = st["x"].view(-1, H + 2 * Hkv, hd)[:, H + Hkv:]
    slots = st["slots"].long()
    base = ((slots // page)[:, None] * Hkv + torch.arange(Hkv, device="cuda")[None, :]) * (page * hd)
    ko, vo = k_offsets(page, hd).cuda()[slots % page], v_offsets(page, hd).cuda()[slots % page]
    st["k"].view(-1)[base[:, :, None] + ko[:, None, :]] = k
    st["v"].view(-1)[base[:, :, None] + vo[:, None, :]] = v
    return {"q": q, "k": st["k"], "v": st["v"]}


def _gathered(pages, table, n, offsets, page, head_dim):
    """[kv_heads, n, head_dim] in 32 bits: the first n keys of a request."""
    t = pages[table[:-(-n // page)]].float()
    t = t[:, :, offsets.view(-1)].view(t.shape[0], t.shape[1], page, head_dim)
    return t.transpose(0, 1).reshape(t.shape[1], -1, head_dim)[:, :n]


def _plain_attend(st):
    H, Hkv, hd, page = st["heads"], st["kv_heads"], st["head_dim"], st["page"]
    group, out, r0 = H // Hkv, torch.empty_like(st["q"]), 0
    ko, vo = k_offsets(page, hd).cuda(), v_offsets(page, hd).cuda()
    for b, (start, count, n) in enumerate(zip(st["starts"], st["counts"], st["lens"])):
        k = _gathered(st["k"], st["table"][b], n, ko, page, hd)
        v = _gathered(st["v"], st["table"][b], n, vo, page, hd)
        q = st["q"][r0:r0 + count].float().view(count, Hkv, group, hd)
        q = q.permute(1, 2, 0, 3).reshape(Hkv, group * count, hd)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(hd))
        if st["causal"]:
            pos = start + torch.arange(count, device="cuda").repeat(group)
            later = torch.arange(n, device="cuda")[None, :] > pos[:, None]
            s = s.masked_fill(later[None], -math.inf)
        e = torch.exp(s - s.amax(dim=-1, keepdim=True))
        o = torch.matmul(e, v.contiguous()) / e.sum(dim=-1, keepdim=True)
        o = o.view(Hkv, group, count, hd).permute(2, 0, 1, 3).reshape(count, H, hd)
        out[r0:r0 + count] = o.to(out.dtype)
        r0 += count
    return {"out": out}


def _own_sample(st):
    from paper_2608_11235_amd import vocab_sample
    token, conf = vocab_sample(st["logits"], st["mask_id"], st["temperature"], st["u"],
                               top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
    return {"token": token, "conf": conf}


def _own_plan(st):
    from paper_2608_11235_amd import cache_plan
    cache, chunk = st["cache"], st["chunk"]
    cache_plan(cache, chunk, reset=st["reset"])
    return {"cu": chunk.cu, "positions": chunk.positions, "slots": chunk.slots,
            "status": chunk.status, "table": cache.table, "len": cache.len, "free": cache.free,
            "n_free": cache.n_free}


def _own_store(st):
    from paper_2608_11235_amd import cache_store
    cache = st["cache"]
    cache_store(cache, 0, st["x"], st["heads"], st["chunk"], rope=st["rope"], q=st["q"])
    return {"q": st["q"], "k": cache.k[0], "v": cache.v[0]}


def _own_attend(st):
    from paper_2608_11235_amd import cache_attention
    cache_attention(st["cache"], 0, st["q"], st["chunk"], st["max_count"], st["max_len"],
                    causal=st["causal"], out=st["out"])
    return {"out": st["out"]}


def run(state):
    """One pass through an operator.  The buffers that a plan or a store updates hold the same
    afterwards however often it is called."""
    kind = state["kind"]
    if own:
        return {"sample": _own_sample, "plan": _own_plan, "store": _own_store,
                "attend": _own_attend}[kind](state)
    return {"sample": _plain_sample, "plan": _plain_plan, "store": _plain_store,
            "attend": _plain_attend}[kind](state)


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    """Bytes and operations of one pass, every input read once and every output written once."""
    if case["kind"] == "sample":
        R, V = case["rows"], case["vocab"]
        par = 4 * (1 + (3 if case["params"] == "mixed" else 1))
        return {"bytes": R * (2 * V + 4 + par + 8), "flops": 4 * R * V}
    _, req = _requests(case, 0)
    B, rows = case["batch"], req["rows"]
    if case["kind"] == "plan":
        taken = int((req["table"] < 0).sum()) if case["reset"] else 0
        touched = int((req["count"] // req["page"] + 1).sum())
        return {"bytes": 4 * (3 * B + touched + 2 * taken + B + 2 * rows + 3 * B + 2),
                "flops": 4 * rows}
    H, Hkv, hd = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "store":
        width = (H + 2 * Hkv) * hd
        distinct = len(np.unique(_row_maps(req)[0]))
        return {"bytes": rows * (4 * width + 8) + distinct * hd * 4, "flops": 3 * rows * (H + Hkv) * hd}
    start, count, n = (req[x].astype(np.int64) for x in ("start", "count", "len"))
    pairs = count * start + count * (count + 1) // 2 if case["causal"] else count * n
    return {"bytes": int(4 * rows * H * hd + 4 * n.sum() * Hkv * hd + 4 * req["table"].size + 12 * B),
            "flops": int(4 * pairs.sum() * H * hd)}


# ---- the same in 64 bits --------------------------------------------------------------------------
def _exact_sample(case, seed):
    if case["rows"] * case["vocab"] > 60_000_000:
        return None
    st = _prepare_sample(case, seed)
    x = st["logits"].double().cpu().numpy()
    par = {k: None if st[k] is None else st[k].double().cpu().numpy()
           for k in ("temperature", "top_k", "top_p", "min_p", "u")}
    ids = np.delete(np.arange(x.shape[1]), st["mask_id"])
    token, conf = np.empty(len(x), np.int32), np.empty(len(x))
    for r, row in enumerate(x):
        l = row[ids]
        order = np.argsort(-l, kind="stable")
        l, who = l[order], ids[order]
        n = int(np.sum(l > -np.inf))
        l, who = l[:n] - l[0], who[:n]
        pick, T = 0, par["temperature"][r]
        if T > 0:
            w = np.exp(l / T)
            if par["top_k"] is not None and par["top_k"][r] > 0:
                w = w[:int(par["top_k"][r])]
            sums, m = np.cumsum(w), len(w)
            if par["top_p"] is not None and par["top_p"][r] < 1:
                m = min(m, 1 + int(np.searchsorted(sums, par["top_p"][r] * sums[-1], side="left")))
            if par["min_p"] is not None and par["min_p"][r] > 0:
                m = min(m, max(1, int(np.sum(w >= par["min_p"][r]))))
            pick = min(int(np.searchsorted(sums[:m], par["u"][r] * sums[m - 1], side="right")), m - 1)
        token[r] = who[pick]
        conf[r] = math.exp(l[pick]) / np.exp(l).sum()
    return {"token": torch.from_numpy(token), "conf": torch.from_numpy(conf)}


def _exact_plan(case, seed):
    """Request by request: pages popped from the stack, rows appended."""
    _, req = _requests(case, seed)
    table, length, page = req["table"].copy(), req["len"].copy(), req["page"]
    free, n_free = req["free"].copy(), int(req["n_free"][0])
    if case["reset"]:
        length[:] = 0
        free, n_free = np.arange(req["n_pages"], dtype=np.int32)[::-1].copy(), req["n_pages"]
    cu, positions, slots = [0], [], []
    for b in range(case["batch"]):
        lo, hi = int(req["start"][b]), int(req["start"][b] + req["count"][b])
        for j in range(-(-int(length[b]) // page), -(-hi // page)):
            n_free -= 1
            table[b, j] = free[n_free]
        length[b] = max(length[b], hi)
        for p in range(lo, hi):
            positions.append(p)
            slots.append(int(table[b, p // page]) * page + p % page)
        cu.append(len(positions))
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32)  # noqa: E731
    return {"cu": i32(cu), "positions": i32(positions), "slots": i32(slots),
            "status": i32(np.zeros(case["batch"])), "table": i32(table), "len": i32(length),
            "free": i32(free), "n_free": i32([n_free])}


def _plain_inputs(fn, case, seed):
    global own
    was, own = own, False
    try:
        return fn(case, seed)
    finally:
        own = was


def _exact_store(case, seed):
    """Rotation as a complex product, token by token of a page's offsets."""
    st = _plain_inputs(_prepare_store, case, seed)
    H, Hkv, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    x = st["x"].double().view(-1, H + 2 * Hkv, hd)
    turn = torch.view_as_complex(st["rope"].double())[st["positions"].long()][:, None, :]
    z = torch.complex(x[:, :H + Hkv, :hd // 2], x[:, :H + Hkv, hd // 2:]) * turn
    qk = torch.cat([z.real, z.imag], dim=-1)
    where = st["slots"].long()
    out = {"q": qk[:, :H]}
    for name, vals, offs in (("k", qk[:, H:], k_offsets(page, hd)),
                             ("v", x[:, H + Hkv:], v_offsets(page, hd))):
        pages = st[name].double()
        for p in range(page):
            sel = where % page == p
            pages[(where[sel] // page)[:, None, None], torch.arange(Hkv, device="cuda")[None, :, None],
                  offs[p].cuda()[None, None, :]] = vals[sel]
        out[name] = pages
    return out


def _exact_attend(case, seed):
    """Query head by query head in 64 bits."""
    st = _plain_inputs(_prepare_attend, case, seed)
    H, Hkv, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    if work(case)["flops"] > 5e11:
        return None
    natural = {}
    for name, offs in (("k", k_offsets(page, hd)), ("v", v_offsets(page, hd))):
        back = torch.empty(page * hd, dtype=torch.long)
        back[torch.arange(page * hd)] = offs.view(-1)
        natural[name] = torch.index_select(st[name], 2, back.cuda()).view(-1, Hkv, page, hd)
    out, r0 = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda"), 0
    for b, (start, count, n) in enumerate(zip(st["starts"], st["counts"], st["lens"])):
        used = st["table"][b][:-(-n // page)]
        for h in range(H):
            k, v = (natural[x][used, h * Hkv // H].reshape(-1, hd)[:n].double() for x in ("k", "v"))
            score = st["q"][r0:r0 + count, h].double() @ k.T / math.sqrt(hd)
            if case["causal"]:
                seen = torch.arange(n, device="cuda") <= start + torch.arange(count, device="cuda")[:, None]
                score[~seen] = -math.inf
            out[r0:r0 + count, h] = torch.softmax(score, dim=-1) @ v
        r0 += count
    return {"out": out}


def exact(case, seed):
    return {"sample": _exact_sample, "plan": _exact_plan, "store": _exact_store,
            "attend": _exact_attend}[case["kind"]](case, seed)
