"""The work that the performance of 8-bit products and of beam search is measured on.

Four operators take a cached decode to 8-bit weights and to several beams a request:

    quantize  rows of activations or weights into 8-bit floating point (e4m3), each 128 columns of a
              row with a power of two as their scale
    product   activations times weights, both in that form, into bf16 or float32
    beam      the best continuations of a request's beams over beams and vocabulary
    reorder   the paged K and V of every beam follow its parent: full pages are shared by counts, the
              last, partly filled page is copied

`run` computes them in elementary torch operations, or calls the package's operators.  8-bit rows are
held in the order of the package's matrix operands; `_packed` and `_unpacked` say where.
"""
import math

import numpy as np
import torch

own = False


# ---- the cases ------------------------------------------------------------------------------
def _quantize(name, rows, cols, dtype, pad):
    return {"name": name, "kind": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "pad": pad}


def _product(name, rows, outs, cols, dtype, bias):
    return {"name": name, "kind": "product", "rows": rows, "outs": outs, "cols": cols,
            "dtype": dtype, "bias": bias}


def _beam(name, batch, beams, width, vocab, ld, done, sigma):
    return {"name": name, "kind": "beam", "batch": batch, "beams": beams, "width": width,
            "vocab": vocab, "ld": ld, "done": done, "sigma": sigma}


def _reorder(name, batch, beams, layers, kv_heads, head_dim, page, prompt, new):
    return {"name": name, "kind": "reorder", "batch": batch, "beams": beams, "layers": layers,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "prompt": prompt, "new": new}


def listed():
    return [
        # the active block of one LLaDA-8B sequence before its projections: latency
        _quantize("quantize_block", 32, 4096, "bf16", 0),
        # the MLP's inner rows of eight Dream-7B canvases: the largest
        _quantize("quantize_canvas", 4096, 18944, "bf16", 0),
        # the tiny model's gate rows for its block: latency alone
        _product("product_tiny", 16, 688, 256, "bf16", False),
        # gate and up of LLaDA-8B for one active block: a stream of 100 MB of weights
        _product("product_block", 32, 24576, 4096, "bf16", False),
        # ragged in every dimension, with a bias, kept in 32 bits
        _product("product_odd", 333, 1531, 1000, "f32", True),
        # gate and up of Dream-7B for eight canvases: the largest, matrix instructions
        _product("product_canvas", 4096, 37888, 3584, "bf16", False),
        # one request of four beams over the tiny model's vocabulary: latency alone
        _beam("beam_tiny", 1, 4, 4, 2048, 2048, False, 2.5),
        # 48 requests of five beams, a vocabulary of odd size in padded rows, some beams finished
        _beam("beam_odd", 48, 5, 10, 50257, 50261, True, 2.0),
        # 128 requests of eight beams over Dream-7B's vocabulary, twice as many candidates: the largest
        _beam("beam_batch", 128, 8, 16, 152064, 152064, False, 1.5),
        # four beams of the tiny model after a short prompt: latency alone
        _reorder("reorder_tiny", 1, 4, 2, 4, 64, 32, 40, 20),
        # eight requests of four beams, Dream-7B heads and layers, behind prompts of up to 1024 tokens
        _reorder("reorder_step", 8, 4, 28, 4, 128, 64, 1024, 200),
        # six requests of four beams, LLaDA-8B heads and layers: the largest copies
        _reorder("reorder_wide", 6, 4, 32, 32, 128, 64, 96, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 to 4096 rows of 64 to 18944 columns; products of 1 to 4096 rows with 16 to
    37888 weight rows; 1 to 128 requests of 1 to 8 beams over 500 to 152064 logits; pages of 32 to 256
    of up to 32 layers and kv heads."""
    kind = rng.choice(["quantize", "product", "product", "product", "beam", "beam", "reorder"])
    if kind == "quantize":
        cols = _log_int(rng, 64, 18944)
        case = _quantize("", _log_int(rng, 1, 4096), cols, rng.choice(["bf16", "bf16", "f32"]),
                         rng.choice([0, 0, 1, 8]))
        if case["rows"] * cols > 38_000_000:
            case["dtype"] = "bf16"
    elif kind == "product":
        rows = _log_int(rng, 1, 4096)
        outs, cols = _log_int(rng, 16, 37888), _log_int(rng, 64, 18944)
        while outs * cols > 140_000_000 or rows * outs * cols > 5.5e11:
            outs = (outs + 1) // 2
        case = _product("", rows, outs, cols, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.4)
    elif kind == "beam":
        batch, beams = _log_int(rng, 1, 128), rng.choice([1, 2, 3, 4, 5, 8])
        vocab = _log_int(rng, 500, 152064)
        case = _beam("", batch, beams, beams * rng.choice([1, 2]), vocab,
                     vocab + rng.choice([0, 0, 1, 3, 8, 64]), rng.random() < 0.5, rng.uniform(0.7, 4.0))
    else:
        beams, page = rng.choice([2, 3, 4, 6, 8]), rng.choice([32, 64, 128, 256])
        kv_heads, head_dim, layers = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([64, 128]), rng.choice([1, 4, 16, 28, 32])
        prompt, new, batch = _log_int(rng, 1, 2048), _log_int(rng, 1, 256), _log_int(rng, 1, 32)
        # the pool fits 1.2 GB
        each = layers * kv_heads * head_dim * 4 * (prompt + page + beams * (new + page))
        while each > 1.2e9:
            layers, each = (layers + 1) // 2, each / 2
        case = _reorder("", max(1, min(batch, int(1.2e9 // each))), beams, layers, kv_heads, head_dim, page,
                        prompt, new)
    del case["name"]
    return case


# ---- 8-bit rows: what they are, and the order they are held in -------------------------------------
def _blocks(x):
    """[R16, 16, nk, 128] float32: rows and columns padded with zeros to multiples of 16 and 128."""
    R, K = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -K % 128, 0, -R % 16))
    return x.view(x.shape[0] // 16, 16, -1, 128)


def _as_8bit(x):
    """(values e4m3 [R16, 16, nk, 128], scales int64 [R16, 16, nk], the power of two's exponent + 127).
    The scale is the least power of two, no less than 2^-127, with which 448 reaches the block's largest
    finite magnitude; a block of zeros has 1."""
    b = _blocks(x)
    most = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax(dim=-1)
    bits = most.view(torch.int32).long()
    e = (bits >> 23) - 135 + ((bits & 0x7fffff) > 0x600000)
    e = torch.where(bits == 0, torch.zeros_like(e), e.clamp(min=-127))
    q = torch.ldexp(b, -e[..., None].int()).to(torch.float8_e4m3fn)
    return q, e + 127


def _grouped(s):
    """Scales [R16, 16, nk] as [R16, 16, ceil(nk / 4), 4] uint8, the blocks past the last one with 1."""
    return torch.nn.functional.pad(s, (0, -s.shape[-1] % 4), value=127).to(torch.uint8).view(*s.shape[:2], -1, 4)


def _packed(q, s):
    """The buffers that hold them: values of 16 rows and 128 columns are 2 KB, byte
    (k / 64) 1024 + (k / 16 % 4) 256 + r 16 + k % 16 of them row r, column k, blocks of a row group one
    after another; scales of 16 rows and four blocks are 64 bytes, byte 4 r + block."""
    q = q.view(torch.uint8).view(q.shape[0], 16, q.shape[2], 2, 4, 16).permute(0, 2, 3, 4, 1, 5)
    return q.reshape(-1), _grouped(s).permute(0, 2, 1, 3).reshape(-1)


def _unpacked(data, scale, rows, cols):
    """Float32 [rows, cols] of what the buffers hold."""
    R16, nk = -(-rows // 16), -(-cols // 128)
    q = data.view(torch.float8_e4m3fn).float().view(R16, nk, 8, 16, 16)
    s = scale.view(R16, -1, 16, 4).permute(0, 1, 3, 2).reshape(R16, -1, 1, 16, 1)[:, :nk]
    x = torch.ldexp(q, s.int() - 127)
    return x.permute(0, 3, 1, 2, 4).reshape(R16 * 16, nk * 128)[:rows, :cols]


def _shown(data, scale, rows, cols):
    """The buffers in the order of rows and columns, without moving them."""
    R16, nk = -(-rows // 16), -(-cols // 128)
    return {"values": data.view(torch.float8_e4m3fn).view(R16, nk, 2, 4, 16, 16).permute(0, 4, 1, 2, 3, 5),
            "scales": scale.view(R16, -1, 16, 4).permute(0, 2, 1, 3)}


# ---- inputs ---------------------------------------------------------------------------------
def _dev(x, dtype=None):
    x = torch.as_tensor(np.ascontiguousarray(x)).cuda()
    return x if dtype is None else x.to(dtype)


def _activations(gen, rows, cols):
    """N(0, 1) rows of differing size with a few columns that stand out, as residual streams have."""
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device="cuda"))
    loud = torch.randint(0, cols, (max(1, cols // 500),), generator=gen, device="cuda")
    x[:, loud] *= 30.0
    return x


def _prepare_quantize(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = _activations(gen, case["rows"], case["cols"] + case["pad"])
    return {"kind": "quantize", "x": x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)[:, :case["cols"]]}


def _prepare_product(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    M, N, K = case["rows"], case["outs"], case["cols"]
    st = {"kind": "product", "rows": M, "outs": N, "cols": K,
          "dtype": torch.bfloat16 if case["dtype"] == "bf16" else torch.float32, "bias": None}
    a = _packed(*_as_8bit(_activations(gen, M, K).to(torch.bfloat16)))
    w = _packed(*_as_8bit(0.02 * torch.randn((N, K), generator=gen, device="cuda")))
    if case["bias"]:
        st["bias"] = torch.randn(N, generator=gen, device="cuda")
    if own:
        from paper_2608_11235_amd import Rows8
        for name, (data, scale), rows in (("a", a, M), ("w", w, N)):
            st[name] = Rows8(rows, K)
            st[name].data.copy_(data)
            st[name].scale.copy_(scale)
    else:
        st.update(a=a, w=w)
    return st


def _prepare_beam(case, seed):
    """Logits N(0, sigma) with a spike of up to 12 in most rows; banned ids hold bf16's lowest number or
    -inf in some; running scores of a few dozen tokens, one beam in ten unused (-inf)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    B, K, V, ld = case["batch"], case["beams"], case["vocab"], case["ld"]
    R = B * K
    x = torch.empty((R, ld), dtype=torch.bfloat16, device="cuda")
    for r0 in range(0, R, 512):
        n = min(512, R - r0)
        y = torch.randn((n, ld), generator=gen, device="cuda") * case["sigma"]
        y[torch.arange(n, device="cuda"), _dev(rng.integers(0, V, size=n))] += \
            _dev(rng.uniform(0.0, 12.0, size=n).astype(np.float32))
        x[r0:r0 + n] = y
    for r in range(0, R, 16):
        x[r, 5:V // 50] = -math.inf if r % 32 else torch.finfo(torch.bfloat16).min
    score = -rng.uniform(5.0, 12.0, size=(B, K))
    score[rng.random((B, K)) < 0.1] = -math.inf
    score[:, 0] = -rng.uniform(5.0, 12.0, size=B)
    done = rng.random((B, K)) < 0.2
    return {"kind": "beam", "logits": x[:, :V], "mask_id": V - V // 1000 - 1, "beams": K, "width": case["width"],
            "score": _dev(score.astype(np.float32)), "done": _dev(done.astype(np.uint8)) if case["done"] else None,
            "done_token": V // 3}


def _beams_of(case, seed):
    """Pages of beams in mid-search on the host: a request's beams share the full pages of its prompt and
    hold the rest themselves; parents drawn among the request's own beams."""
    shape = np.random.default_rng([case["batch"], case["beams"], case["page"], case["prompt"], case["new"]])
    B, K, P = case["batch"], case["beams"], case["page"]
    prompt = shape.integers(max(1, case["prompt"] // 2), case["prompt"] + 1, size=B)
    length = prompt + shape.integers(max(1, case["new"] // 2), case["new"] + 1, size=B)
    pick = shape.integers(0, K, size=(B, K))  # half of the beams or so live on
    shared, held = prompt // P, -(-length // P)
    rng = np.random.default_rng(seed)
    n_pages = int((shared + K * (held - shared)).sum()) + 5
    order, at = rng.permutation(n_pages), 0
    table = np.full((B, K, int(held.max())), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    for b in range(B):
        table[b, :, :shared[b]] = order[at:at + shared[b]]
        refs[order[at:at + shared[b]]] = K
        at += shared[b]
        own_pages = K * (held[b] - shared[b])
        table[b, :, shared[b]:held[b]] = order[at:at + own_pages].reshape(K, -1)
        refs[order[at:at + own_pages]] = 1
        at += own_pages
    free = np.zeros(n_pages, np.int32)
    free[:n_pages - at] = order[at:]
    who = np.stack([rng.permutation(K) for _ in range(B)])  # the seed says which beam is which
    parent = np.arange(B)[:, None] * K + np.take_along_axis(who, pick, 1)
    i32 = np.int32
    return {"table": table.reshape(B * K, -1), "len": np.repeat(length, K).astype(i32), "refs": refs, "free": free,
            "n_free": np.array([n_pages - at], i32), "parent": parent.reshape(-1).astype(i32), "n_pages": n_pages}


_PAGES = ("table", "len", "refs", "free", "n_free")


def _prepare_reorder(case, seed):
    req = _beams_of(case, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    P, hd, Hkv = case["page"], case["head_dim"], case["kv_heads"]
    st = {"kind": "reorder", "page": P, "group": 32 * hd, "parent": _dev(req["parent"])}
    shape = (case["layers"], req["n_pages"], Hkv, P * hd)
    if own:
        from paper_2608_11235_amd import KVCache
        cache = st["cache"] = KVCache(case["layers"], req["n_pages"], Hkv, hd, P, case["batch"] * case["beams"],
                                      req["table"].shape[1], shared=True)
        for name in _PAGES:
            getattr(cache, name).copy_(_dev(req[name]))
        k, v = cache.k, cache.v
    else:
        st.update({name: _dev(req[name]) for name in _PAGES})
        k, v = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        st.update(k=k, v=v)
    for pages in (k, v):
        for layer in pages:
            layer.copy_(torch.randn(shape[1:], generator=gen, device="cuda"))
    return st


def prepare(case, seed):
    return {"quantize": _prepare_quantize, "product": _prepare_product, "beam": _prepare_beam,
            "reorder": _prepare_reorder}[case["kind"]](case, seed)


# ---- one pass ---------------------------------------------------------------------------------
def _plain_quantize(st):
    q, s = _as_8bit(st["x"])
    return {"values": q.view(*q.shape[:3], 2, 4, 16), "scales": _grouped(s)}


def _plain_product(st):
    a = _unpacked(*st["a"], st["rows"], st["cols"])
    w = _unpacked(*st["w"], st["outs"], st["cols"])
    out = torch.mm(a, w.t())
    if st["bias"] is not None:
        out = out + st["bias"]
    return {"out": out.to(st["dtype"])}


def _ordered(logits):
    """Whole numbers in the order of the bf16 logits (no NaN), zeros alike."""
    bits = (logits + 0.0).view(torch.int16).long() & 0xffff
    bits = torch.where(bits == 0x8000, torch.zeros_like(bits), bits)
    return torch.where(bits >= 0x8000, 0xffff - bits, bits + 0x8000)


def _plain_beam(st):
    """The best of every row by (logit, id), then the best of a request's rows by score; in 64 bits,
    since a difference in the last place orders two candidates."""
    logits, K, W, mask_id = st["logits"], st["beams"], st["width"], st["mask_id"]
    R, V = logits.shape
    x = logits.clone()
    x[:, mask_id] = -math.inf
    m = x.amax(dim=1, keepdim=True).double()
    lse = m[:, 0] + torch.log(torch.exp(x.double() - m).sum(dim=1))
    key = (_ordered(x) << 18) + (V - 1 - torch.arange(V, device="cuda"))
    n = min(W, V)
    at = V - 1 - (torch.topk(key, n, dim=1).values & ((1 << 18) - 1))
    best = torch.gather(x, 1, at).double()
    score = st["score"].view(-1).double()
    cand = score[:, None] + (best - lse[:, None])
    if st["done"] is not None:
        over = st["done"].view(-1, 1) != 0
        first = torch.arange(n, device="cuda")[None, :] == 0
        cand = torch.where(over, torch.where(first, score[:, None], -math.inf), cand)
        at = torch.where(over, torch.full_like(at, st["done_token"]), at)
    row = torch.arange(R, device="cuda")[:, None].expand(R, n)
    top, order = torch.sort(cand.reshape(R // K, K * n), dim=1, descending=True, stable=True)
    top, order = top[:, :W], order[:, :W]
    none = top == -math.inf
    take = lambda t: torch.where(none, -1, torch.gather(t.reshape(R // K, K * n), 1, order)).int()  # noqa: E731
    return {"token": take(at), "parent": take(row), "score": top.float()}


def _plain_reorder(st):
    """Counts of children, pages given back in the order of their holders, copies of partly filled pages
    for all but a parent's first child, then the tables."""
    table, length, refs, free, n_free = (st[n] for n in _PAGES)
    B, most = table.shape
    P, n_pages = st["page"], refs.shape[0]
    p, j = st["parent"].long(), torch.arange(B, device="cuda")
    L = length.long()
    held, full = (L + P - 1) // P, L // P
    i = torch.arange(most, device="cuda")[None, :]
    pages = table.long().clamp(0, n_pages - 1)
    holds, whole = i < held[:, None], i < full[:, None]
    children = torch.zeros(B, dtype=torch.long, device="cuda").index_add_(0, p, torch.ones_like(p))
    first = torch.full((B,), B, device="cuda").scatter_reduce_(0, p, j, "amin")
    copies = (first[p] != j) & (held[p] > full[p])
    # the pages that nobody holds any more
    change = torch.where(whole, children[:, None] - 1, torch.where(children[:, None] > 0, 0, -1))
    change = torch.where(holds, change, torch.zeros_like(change))
    left = refs.long().index_add(0, pages.view(-1), change.view(-1))
    flat = (j[:, None] * most + i).view(-1)
    drops = (holds & (children[:, None] == 0)).view(-1) & (left[pages.view(-1)] == 0)
    lowest = torch.full((n_pages,), B * most, device="cuda").scatter_reduce_(
        0, pages.view(-1), torch.where(drops, flat, B * most), "amin")
    gives = drops & (lowest[pages.view(-1)] == flat)
    stack = torch.cat([free, free.new_zeros(1)])
    at = torch.where(gives, n_free.long() + torch.cumsum(gives, 0) - 1, n_pages)
    stack.scatter_(0, at, pages.view(-1).int())
    there = n_free.long() + gives.sum()
    # pages for the copies
    rank = torch.cumsum(copies, 0)
    refused = copies & (rank > there)
    copies = copies & ~refused
    fresh = stack[(there - rank).clamp(0, n_pages)].long()
    kept = torch.zeros(B, dtype=torch.long, device="cuda").index_add_(0, p, (~refused).long())
    change = torch.where(whole, kept[:, None] - 1, torch.where(kept[:, None] > 0, 0, -1))
    left = refs.long().index_add(0, pages.view(-1), torch.where(holds, change, 0).view(-1))
    rows = copies.nonzero()[:, 0]
    src, dst, par = pages[p[rows], full[p[rows]]], fresh[rows], p[rows]
    left[dst] = 1
    groups = (L[par] % P + 31) // 32
    used = torch.arange(P // 32, device="cuda")[None, :] < groups[:, None]
    for x in (st["k"], st["v"]):
        y = x.view(*x.shape[:3], P // 32, st["group"])
        y[:, dst] = torch.where(used[None, :, None, :, None], y[:, src], y[:, dst])
    new = torch.where(i < torch.where(refused, 0, held[p])[:, None], table[p], table)
    new[rows, full[par]] = dst.int()
    table.copy_(new)
    length.copy_(torch.where(refused, 0, L[p]))
    refs.copy_(left)
    free.copy_(stack[:n_pages])
    n_free.copy_(there - copies.sum())
    return {"status": torch.where(refused, -3, 0).int(), **{n: st[n] for n in _PAGES}, "k": st["k"], "v": st["v"]}


def _own_quantize(st):
    from paper_2608_11235_amd import quantize_rows
    q = quantize_rows(st["x"])
    return _shown(q.data, q.scale, *st["x"].shape)


def _own_product(st):
    from paper_2608_11235_amd import rows8_product
    return {"out": rows8_product(st["a"], st["w"], bias=st["bias"], dtype=st["dtype"])}


def _own_beam(st):
    from paper_2608_11235_amd import vocab_beam
    token, parent, score = vocab_beam(st["logits"], st["beams"], st["mask_id"], st["score"], width=st["width"],
                                      done=st["done"], done_token=st["done_token"])
    return {"token": token, "parent": parent, "score": score}


def _own_reorder(st):
    from paper_2608_11235_amd import cache_reorder
    cache = st["cache"]
    status = cache_reorder(cache, st["parent"])
    return {"status": status, **{n: getattr(cache, n) for n in _PAGES}, "k": cache.k, "v": cache.v}


def run(state):
    """One pass through an operator.  A reorder leaves beams of the same lengths, so that the next one by
    the same parents copies as much."""
    kind = state["kind"]
    if own:
        return {"quantize": _own_quantize, "product": _own_product, "beam": _own_beam,
                "reorder": _own_reorder}[kind](state)
    return {"quantize": _plain_quantize, "product": _plain_product, "beam": _plain_beam,
            "reorder": _plain_reorder}[kind](state)


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    """Bytes and operations of one pass, every input read once and every output written once."""
    kind = case["kind"]
    if kind == "quantize":
        R, K = case["rows"], case["cols"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": R * K * (size + 1) + R * -(-K // 128), "flops": 2 * R * K}
    if kind == "product":
        M, N, K = case["rows"], case["outs"], case["cols"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": (M + N) * (K + -(-K // 128)) + M * N * size + (4 * N if case["bias"] else 0),
                "flops": 2 * M * N * K}
    if kind == "beam":
        R, V = case["batch"] * case["beams"], case["vocab"]
        return {"bytes": R * (2 * V + 4 + (1 if case["done"] else 0)) + 12 * case["batch"] * case["width"],
                "flops": 4 * R * V}
    req = _beams_of(case, 0)
    P, parent, n = case["page"], req["parent"], req["len"]
    held = -(-n // P)
    again = np.ones(len(parent), bool)
    again[np.unique(parent, return_index=True)[1]] = False
    groups = np.where(again, (n[parent] % P + 31) // 32, 0).sum()
    each = case["layers"] * case["kv_heads"] * 32 * case["head_dim"] * 4
    return {"bytes": int(2 * groups * each + 4 * (held.sum() * 2 + 2 * req["n_pages"] + 4 * len(parent))), "flops": 0}


# ---- the same in 64 bits --------------------------------------------------------------------------
def _plain_inputs(fn, case, seed):
    global own
    was, own = own, False
    try:
        return fn(case, seed)
    finally:
        own = was


def _exact_quantize(case, seed):
    """Scales from the logarithm of the largest magnitude, values by rounding to multiples of their step."""
    x = _prepare_quantize(case, seed)["x"].double()
    R, K = x.shape
    b = torch.zeros((-(-R // 16) * 16, -(-K // 128) * 128), dtype=torch.float64, device="cuda")
    b[:R, :K] = x
    b = b.view(b.shape[0] // 16, 16, -1, 128)
    part, power = torch.frexp(b.abs().amax(dim=-1, keepdim=True) / 448)
    e = (power - (part == 0.5).int()).clamp(min=-127)
    e = torch.where(part == 0, torch.zeros_like(e), e)
    y = b * torch.exp2(-e.double())
    step = torch.exp2((torch.frexp(y).exponent - 1).clamp(min=-6).double() - 3)
    scales = torch.full((b.shape[0], 16, -(-b.shape[2] // 4) * 4), 127, dtype=torch.uint8, device="cuda")
    scales[..., :b.shape[2]] = (e[..., 0] + 127).to(torch.uint8)
    return {"values": (torch.round(y / step) * step).view(*b.shape[:3], 2, 4, 16),
            "scales": scales.view(b.shape[0], 16, -1, 4)}


def _exact_product(case, seed):
    """Entry by entry of the buffers' order, products in 64 bits."""
    st = _plain_inputs(_prepare_product, case, seed)

    def natural(data, scale, rows):
        r = torch.arange(rows, device="cuda")[:, None]
        k = torch.arange(case["cols"], device="cuda")[None, :]
        nk = -(-case["cols"] // 128)
        at = ((r // 16) * nk + k // 128) * 2048 + (k % 128 // 64) * 1024 + (k // 16 % 4) * 256 + (r % 16) * 16 + k % 16
        sc = ((r // 16) * -(-nk // 4) + k // 512) * 64 + (r % 16) * 4 + k // 128 % 4
        return data[at].view(torch.float8_e4m3fn).double() * torch.exp2(scale[sc].double() - 127)

    out = natural(*st["a"], case["rows"]) @ natural(*st["w"], case["outs"]).t().contiguous()
    return {"out": out if st["bias"] is None else out + st["bias"].double()}


def _exact_beam(case, seed):
    """All of a request's candidates sorted at once, request by request."""
    st = _prepare_beam(case, seed)
    K, W, V = case["beams"], case["width"], case["vocab"]
    out = {"token": [], "parent": [], "score": []}
    for b in range(case["batch"]):
        rows = slice(b * K, (b + 1) * K)
        x = st["logits"][rows].double()
        x[:, st["mask_id"]] = -math.inf
        s = st["score"][b].double()[:, None] + torch.log_softmax(x, dim=1)
        if st["done"] is not None:
            for k in range(K):
                if int(st["done"][b, k]):
                    s[k] = -math.inf
                    s[k, st["done_token"]] = st["score"][b, k].double()
        s, at = torch.sort(s.view(-1), descending=True, stable=True)
        s, at = s[:W], at[:W]
        gone = s == -math.inf
        out["token"].append(torch.where(gone, -1, at % V).int())
        out["parent"].append(torch.where(gone, -1, b * K + at // V).int())
        out["score"].append(s)
    return {n: torch.stack(v) for n, v in out.items()}


def _exact_reorder(case, seed):
    """Beam by beam with lists of pages."""
    req = _beams_of(case, seed)
    st = _plain_inputs(_prepare_reorder, case, seed)
    P, parent, B = case["page"], req["parent"], len(req["parent"])
    table, refs = req["table"].copy(), req["refs"].copy()
    stack = list(req["free"][:int(req["n_free"][0])])
    free = req["free"].copy()
    old = [list(table[b, :-(-int(req["len"][b]) // P)]) for b in range(B)]
    new, length, moves, seen = [], np.zeros(B, np.int32), [], set()
    wants = []
    for b in range(B):
        p = int(parent[b])
        n, mine = int(req["len"][p]), list(old[p])
        if p in seen and n % P:
            wants.append((b, len(mine) - 1))
        seen.add(p)
        new.append(mine)
        length[b] = n
    count = np.zeros(req["n_pages"], np.int64)
    for b, mine in enumerate(new):
        for i, page in enumerate(mine):
            if (b, i) not in wants:
                count[page] += 1
    for b in range(B):
        for page in old[b]:
            if count[page] == 0 and refs[page] > 0:
                refs[page] = 0
                free[len(stack)] = page
                stack.append(page)
    for b, i in wants:
        page = stack.pop()
        moves.append((new[b][i], page, (int(length[b]) % P + 31) // 32))
        new[b][i] = page
        count[page] = 1
    for b, mine in enumerate(new):
        table[b, :len(mine)] = mine
    for x in (st["k"], st["v"]):
        y = x.view(*x.shape[:3], P // 32, -1)
        for src, dst, groups in moves:
            y[:, int(dst), :, :groups] = y[:, int(src), :, :groups]
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32)  # noqa: E731
    return {"status": i32(np.zeros(B)), "table": i32(table), "len": i32(length), "refs": i32(count), "free": i32(free),
            "n_free": i32([len(stack)]), "k": st["k"], "v": st["v"]}


def exact(case, seed):
    return {"quantize": _exact_quantize, "product": _exact_product, "beam": _exact_beam,
            "reorder": _exact_reorder}[case["kind"]](case, seed)
