"""Pythonic wrappers over the C ABI (marshalling only)."""
import ctypes
from typing import Optional
from dataclasses import dataclass

import numpy as np
import torch

from . import _lib
from ._lib import check, ptr, stream_handle

TENSOR_EMBED = 1
TENSOR_LM_HEAD = 2
_LAYER_SLOTS = {"wq": 0, "wk": 1, "wv": 2, "wo": 3, "wg": 4, "wu": 5, "wd": 6,
                "bq": 7, "bk": 8, "bv": 9}


_BF16_BITS = (torch.int16, torch.bfloat16, torch.uint16)


def check_device_tensor(t, name, dtypes, numel=None):
    """Refuse what the C ABI would misread: a host or non-contiguous tensor, another element
    type, or fewer elements than the call reads or writes (the library sees only a pointer)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a GPU tensor (got device {t.device})")
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, the call needs {numel}")
    return t


def layer_tensor_id(layer: int, name: str) -> int:
    return 100 + 16 * layer + _LAYER_SLOTS[name]


def model_cfg_from(spec) -> _lib.ModelCfg:
    """Build the C struct from any object carrying the backbone fields."""
    return _lib.ModelCfg(spec.n_layers, spec.d_model, spec.n_heads, spec.n_kv_heads,
                         spec.head_dim, spec.ffn_dim, spec.vocab, spec.mask_id,
                         int(bool(spec.qkv_bias)), spec.rms_eps, spec.rope_theta,
                         spec.logit_scale, float(getattr(spec, "init_std", 0.02)))


@dataclass
class Sched:
    block_len: int = 32
    steps_per_block: int = 32
    eos_id: Optional[int] = None   # EOS-aware controller when set

    def c(self):
        return _lib.SchedCfg(self.block_len, self.steps_per_block,
                             0 if self.eos_id is None else 1,
                             0 if self.eos_id is None else int(self.eos_id))


@dataclass
class Gate:
    delta_p: float = 0.65
    m_req: int = 1
    enabled: bool = True
    persist_scope: int = 0

    def c(self):
        return _lib.GateCfg(self.delta_p, self.m_req, int(self.enabled), self.persist_scope)


class DecodeState:
    """Device-resident decode state (see cora_state in include/cora.h)."""

    def __init__(self, B, prompt_len, gen_len, n_rows, block_len, device="cuda", passes=True):
        i32, u8 = torch.int32, torch.uint8
        L = prompt_len + gen_len
        self.B, self.prompt_len, self.gen_len, self.block_len = B, prompt_len, gen_len, block_len
        self.tokens = torch.zeros((B, L), dtype=i32, device=device)
        self.unresolved = torch.zeros((B, L), dtype=u8, device=device)
        self.prev_top1 = torch.full((B, L), -1, dtype=i32, device=device)
        self.persist = torch.zeros((B, L), dtype=i32, device=device)
        self.block_idx = torch.zeros(B, dtype=i32, device=device)
        self.step_idx = torch.zeros(B, dtype=i32, device=device)
        self.top1 = torch.zeros((B, n_rows), dtype=i32, device=device)
        self.conf = torch.zeros((B, n_rows), dtype=torch.float32, device=device)
        self.decision = torch.zeros((B, block_len), dtype=u8, device=device)
        self.done = torch.zeros(B, dtype=i32, device=device)
        n_blocks = gen_len // block_len
        self.passes = torch.zeros((B, n_blocks), dtype=i32, device=device) if passes else None

    @classmethod
    def from_host(cls, host: dict, prompt_len, gen_len, n_rows, block_len, device="cuda"):
        """Copy a host state dict (numpy arrays as in seeded_inputs) to the device."""
        B = host["tokens"].shape[0]
        st = cls(B, prompt_len, gen_len, n_rows, block_len, device)
        st.load(host)
        return st

    def load(self, host: dict):
        for name in ("tokens", "unresolved", "prev_top1", "persist", "block_idx", "step_idx"):
            src = torch.from_numpy(np.ascontiguousarray(host[name]))
            getattr(self, name).copy_(src.to(getattr(self, name).dtype))

    def to_host(self) -> dict:
        names = ("tokens", "unresolved", "prev_top1", "persist", "block_idx", "step_idx", "top1",
                 "conf", "decision", "done")
        out = {n: getattr(self, n).cpu().numpy() for n in names}
        if self.passes is not None:
            out["passes"] = self.passes.cpu().numpy()
        return out

    def c(self):
        B, L = self.B, self.prompt_len + self.gen_len
        for name, dt, n in (("tokens", torch.int32, B * L), ("unresolved", torch.uint8, B * L),
                            ("prev_top1", torch.int32, B * L), ("persist", torch.int32, B * L),
                            ("block_idx", torch.int32, B), ("step_idx", torch.int32, B),
                            ("top1", torch.int32, None), ("conf", torch.float32, None),
                            ("decision", torch.uint8, None), ("done", torch.int32, B)):
            check_device_tensor(getattr(self, name), f"state.{name}", (dt,), n)
        if self.passes is not None:
            check_device_tensor(self.passes, "state.passes", (torch.int32,),
                                B * (self.gen_len // self.block_len))
        return _lib.State(ptr(self.tokens), ptr(self.unresolved), ptr(self.prev_top1),
                          ptr(self.persist), ptr(self.block_idx), ptr(self.step_idx),
                          ptr(self.top1), ptr(self.conf), ptr(self.decision), ptr(self.done),
                          ptr(self.passes), self.B, self.prompt_len, self.gen_len)


class Model:
    """Seeded backbone + workspace owned by libcora (weights drawn on the GPU)."""

    def __init__(self, spec, seed: int, max_batch: int, max_seq: int, stream=None):
        lib = _lib.load()
        self.spec, self.seed, self.max_batch, self.max_seq = spec, seed, max_batch, max_seq
        self._cfg = model_cfg_from(spec)
        h = ctypes.c_void_p()
        check(lib.cora_model_create(ctypes.byref(self._cfg), seed, max_batch, max_seq,
                                    stream_handle(stream), ctypes.byref(h)), "cora_model_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            _lib.load().cora_model_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def handle(self):
        return self._h

    def forward_logits(self, tokens, row_begin, n_rows, out=None, stream=None):
        check_device_tensor(tokens, "tokens", (torch.int32,))
        B, L = tokens.shape
        if out is None:
            out = torch.empty((B, n_rows, self.spec.vocab), dtype=torch.int16,
                              device=tokens.device)
        check_device_tensor(out, "out", _BF16_BITS, B * n_rows * self.spec.vocab)
        check(_lib.load().cora_forward_logits(self._h, ptr(tokens), B, L, row_begin, n_rows,
                                               ptr(out), stream_handle(stream)),
              "cora_forward_logits")
        return out

    def denoise_step(self, state: DecodeState, sched: Sched, gate: Gate, stream=None):
        st, sc, gt = state.c(), sched.c(), gate.c()
        check(_lib.load().cora_denoise_step(self._h, ctypes.byref(st), ctypes.byref(sc),
                                             ctypes.byref(gt), stream_handle(stream)),
              "cora_denoise_step")

    def block_decode(self, prompt, gen_len, sched: Sched, gate: Gate, out=None, stream=None):
        check_device_tensor(prompt, "prompt", (torch.int32,))
        B, P = prompt.shape
        if out is None:
            out = torch.empty((B, P + gen_len), dtype=torch.int32, device=prompt.device)
        check_device_tensor(out, "out", (torch.int32,), B * (P + gen_len))
        n_blocks = gen_len // sched.block_len
        passes = np.zeros((B, n_blocks), dtype=np.int32)
        total = ctypes.c_int32(0)
        sc, gt = sched.c(), gate.c()
        check(_lib.load().cora_block_decode(self._h, ptr(prompt), B, P, gen_len, ctypes.byref(sc),
                                             ctypes.byref(gt), ptr(out),
                                             ctypes.c_void_p(passes.ctypes.data),
                                             ctypes.byref(total), stream_handle(stream)),
              "cora_block_decode")
        return out, passes, int(total.value)

    def forward_cached(self, cache, chunk, tokens, max_count=0, max_len=0, causal=False, out=None,
                       stream=None):
        """Logits [chunk.rows, vocab] (bf16 bits) of a planned chunk against the cache, whose pages
        receive the chunk's K and V (cora_forward_cached)."""
        check_device_tensor(tokens, "tokens", (torch.int32,), chunk.rows)
        if out is None:
            out = torch.empty((chunk.rows, self.spec.vocab), dtype=torch.int16, device=tokens.device)
        check_device_tensor(out, "out", _BF16_BITS, chunk.rows * self.spec.vocab)
        _same_device(cache.k, tokens=tokens, out=out)
        ca, pg, ch = cache.c(), cache.pages(), chunk.c(cache)
        check(_lib.load().cora_forward_cached(self._h, ctypes.byref(ca), ctypes.byref(pg), ctypes.byref(ch),
                                               ptr(tokens), max_count, max_len, int(bool(causal)),
                                               ptr(out), stream_handle(stream)), "cora_forward_cached")
        return out

    def copy_tensor(self, tensor_id: int, n_elements: int) -> np.ndarray:
        out = np.empty(n_elements, dtype=np.uint16)
        check(_lib.load().cora_model_copy_tensor(self._h, tensor_id,
                                                  ctypes.c_void_p(out.ctypes.data), out.nbytes),
              "cora_model_copy_tensor")
        return out

    def set_compaction(self, enable: bool):
        check(_lib.load().cora_model_set_compaction(self._h, int(enable)),
              "cora_model_set_compaction")

    def set_timing(self, enable: bool):
        check(_lib.load().cora_model_set_timing(self._h, int(enable)), "cora_model_set_timing")

    def read_timing(self):
        ms, n = ctypes.c_double(0), ctypes.c_int64(0)
        check(_lib.load().cora_model_read_timing(self._h, ctypes.byref(ms), ctypes.byref(n)),
              "cora_model_read_timing")
        return ms.value, n.value

    def device_bytes(self):
        w, ws = ctypes.c_size_t(0), ctypes.c_size_t(0)
        check(_lib.load().cora_model_device_bytes(self._h, ctypes.byref(w), ctypes.byref(ws)),
              "cora_model_device_bytes")
        return w.value, ws.value


def vocab_gate(logits, n_rows, row_begin, V, mask_id, state: DecodeState, k_transfer,
               sched: Sched, gate: Gate, stream=None):
    check_device_tensor(logits, "logits", _BF16_BITS, state.B * n_rows * V)
    st, sc, gt = state.c(), sched.c(), gate.c()
    check(_lib.load().cora_vocab_gate(ptr(logits), n_rows, row_begin, V, mask_id,
                                       ctypes.byref(st), k_transfer, ctypes.byref(sc),
                                       ctypes.byref(gt), stream_handle(stream)),
          "cora_vocab_gate")


def vocab_gate_noalloc(logits, n_rows, row_begin, V, mask_id, state: DecodeState, k_transfer,
                       sched: Sched, gate: Gate, stream=None):
    """cora_vocab_gate_noalloc: vocab_gate without any allocation (split rows, fixed scratch)."""
    check_device_tensor(logits, "logits", _BF16_BITS, state.B * n_rows * V)
    st, sc, gt = state.c(), sched.c(), gate.c()
    check(_lib.load().cora_vocab_gate_noalloc(ptr(logits), n_rows, row_begin, V, mask_id,
                                               ctypes.byref(st), k_transfer, ctypes.byref(sc),
                                               ctypes.byref(gt), stream_handle(stream)),
          "cora_vocab_gate_noalloc")


# ---- sampling --------------------------------------------------------------------------------
def _same_device(first, **others):
    """Refuse tensors of another GPU than `first`'s; None entries are skipped."""
    for name, t in others.items():
        if t is not None and t.device != first.device:
            raise ValueError(f"{name}: on {t.device}, expected {first.device}")


def _sample_rows(R, first, temperature, u, top_k, top_p, min_p):
    f32, i32 = (torch.float32,), (torch.int32,)
    check_device_tensor(temperature, "temperature", f32, R)
    check_device_tensor(u, "u", f32, R)
    for name, t, dt in (("top_k", top_k, i32), ("top_p", top_p, f32), ("min_p", min_p, f32)):
        if t is not None:
            check_device_tensor(t, name, dt, R)
    _same_device(first, temperature=temperature, u=u, top_k=top_k, top_p=top_p, min_p=min_p)
    return _lib.SampleRows(ptr(temperature), ptr(top_k), ptr(top_p), ptr(min_p), ptr(u))


def vocab_sample(logits, mask_id, temperature, u, top_k=None, top_p=None, min_p=None, token=None,
                 conf=None, stream=None):
    """A token per row of the bf16 logits [R, V] and its confidence (cora_vocab_sample).

    temperature, u, top_p, min_p float32 [R], top_k int32 [R]; top_k, top_p and min_p may be None.
    Rows may be strided (logits.stride(1) == 1); mask_id -1 leaves no id out.  Returns
    (token int32 [R], conf float32 [R])."""
    if not isinstance(logits, torch.Tensor):
        raise TypeError(f"logits: expected a torch.Tensor, got {type(logits).__name__}")
    if logits.dim() != 2:
        raise ValueError(f"logits: expected [R, V], got {tuple(logits.shape)}")
    if logits.dtype not in _BF16_BITS:
        raise TypeError(f"logits: dtype {logits.dtype}, expected one of {_BF16_BITS}")
    if not logits.is_cuda:
        raise ValueError(f"logits: must be a GPU tensor (got device {logits.device})")
    R, V = logits.shape
    if (V > 1 and logits.stride(1) != 1) or (R > 1 and logits.stride(0) < V):
        raise ValueError(f"logits: strides {logits.stride()}, expected rows of stride 1 that do not overlap")
    rows = _sample_rows(R, logits, temperature, u, top_k, top_p, min_p)
    if token is None:
        token = torch.empty(R, dtype=torch.int32, device=logits.device)
    if conf is None:
        conf = torch.empty(R, dtype=torch.float32, device=logits.device)
    check_device_tensor(token, "token", (torch.int32,), R)
    check_device_tensor(conf, "conf", (torch.float32,), R)
    _same_device(logits, token=token, conf=conf)
    with torch.cuda.device(logits.device):
        check(_lib.load().cora_vocab_sample(ptr(logits), R, V, logits.stride(0) if R > 1 else V, mask_id,
                                             ctypes.byref(rows), ptr(token), ptr(conf),
                                             stream_handle(stream)), "cora_vocab_sample")
    return token, conf


def vocab_gate_sampled(logits, n_rows, row_begin, V, mask_id, state: DecodeState, k_transfer,
                       sched: Sched, gate: Gate, temperature, u, top_k=None, top_p=None, min_p=None,
                       stream=None):
    """vocab_gate with each row's token drawn as by vocab_sample (cora_vocab_gate_sampled)."""
    check_device_tensor(logits, "logits", _BF16_BITS, state.B * n_rows * V)
    check_device_tensor(state.top1, "state.top1", (torch.int32,), state.B * n_rows)
    check_device_tensor(state.conf, "state.conf", (torch.float32,), state.B * n_rows)
    rows = _sample_rows(state.B * n_rows, logits, temperature, u, top_k, top_p, min_p)
    _same_device(logits, **{"state.tokens": state.tokens})
    st, sc, gt = state.c(), sched.c(), gate.c()
    with torch.cuda.device(logits.device):
        check(_lib.load().cora_vocab_gate_sampled(ptr(logits), n_rows, row_begin, V, mask_id,
                                                   ctypes.byref(st), k_transfer, ctypes.byref(sc),
                                                   ctypes.byref(gt), ctypes.byref(rows),
                                                   stream_handle(stream)), "cora_vocab_gate_sampled")


# ---- paged K/V cache ---------------------------------------------------------------------------
class KVCache:
    """Paged K and V of n_layers layers and the pages that up to `batch` requests hold of them
    (cora_cache and cora_pages in include/cora.h).  Starts empty, all pages free."""

    def __init__(self, n_layers, n_pages, n_kv_heads, head_dim, page_size, batch, max_pages,
                 device="cuda"):
        i32 = torch.int32
        self.n_layers, self.n_pages, self.n_kv_heads = n_layers, n_pages, n_kv_heads
        self.head_dim, self.page_size, self.batch, self.max_pages = head_dim, page_size, batch, max_pages
        shape = (n_layers, n_pages, n_kv_heads, page_size * head_dim)
        self.k = torch.empty(shape, dtype=torch.bfloat16, device=device)
        self.v = torch.empty(shape, dtype=torch.bfloat16, device=device)
        self.table = torch.full((batch, max_pages), -1, dtype=i32, device=device)
        self.len = torch.zeros(batch, dtype=i32, device=device)
        self.free = torch.arange(n_pages - 1, -1, -1, dtype=i32, device=device)
        self.n_free = torch.full((1,), n_pages, dtype=i32, device=device)

    def c(self):
        n = self.n_layers * self.n_pages * self.n_kv_heads * self.page_size * self.head_dim
        check_device_tensor(self.k, "cache.k", _BF16_BITS, n)
        check_device_tensor(self.v, "cache.v", _BF16_BITS, n)
        _same_device(self.k, **{"cache.v": self.v})
        return _lib.Cache(ptr(self.k), ptr(self.v), self.n_layers, self.n_pages, self.n_kv_heads,
                          self.page_size, self.head_dim)

    def pages(self):
        for name, n in (("table", self.batch * self.max_pages), ("len", self.batch),
                        ("free", self.n_pages), ("n_free", 1)):
            check_device_tensor(getattr(self, name), f"cache.{name}", (torch.int32,), n)
            _same_device(self.k, **{f"cache.{name}": getattr(self, name)})
        return _lib.Pages(ptr(self.table), ptr(self.len), ptr(self.free), ptr(self.n_free),
                          self.batch, self.max_pages, self.n_pages, self.page_size)


class Chunk:
    """The rows of one pass: positions [start, start + count) of each request, up to `rows` in all
    (cora_chunk).  The caller fills start and count; cache_plan writes the rest."""

    def __init__(self, batch, rows, device="cuda"):
        i32 = torch.int32
        self.batch, self.rows = batch, rows
        self.start = torch.zeros(batch, dtype=i32, device=device)
        self.count = torch.zeros(batch, dtype=i32, device=device)
        self.cu = torch.zeros(batch + 1, dtype=i32, device=device)
        self.positions = torch.full((rows,), -1, dtype=i32, device=device)
        self.slots = torch.full((rows,), -1, dtype=i32, device=device)
        self.status = torch.zeros(batch, dtype=i32, device=device)

    def c(self, cache):
        if self.batch != cache.batch:
            raise ValueError(f"chunk: {self.batch} requests, the cache has {cache.batch}")
        for name, n in (("start", self.batch), ("count", self.batch), ("cu", self.batch + 1),
                        ("positions", self.rows), ("slots", self.rows), ("status", self.batch)):
            check_device_tensor(getattr(self, name), f"chunk.{name}", (torch.int32,), n)
            _same_device(cache.k, **{f"chunk.{name}": getattr(self, name)})
        return _lib.ChunkRows(ptr(self.start), ptr(self.count), ptr(self.cu), ptr(self.positions),
                              ptr(self.slots), ptr(self.status), self.rows)


def cache_plan(cache: KVCache, chunk: Chunk, reset=False, stream=None):
    """Pages for the chunk and its rows' positions and slots (cora_cache_plan)."""
    pg, ch = cache.pages(), chunk.c(cache)
    with torch.cuda.device(cache.k.device):
        check(_lib.load().cora_cache_plan(ctypes.byref(pg), ctypes.byref(ch), int(bool(reset)),
                                           stream_handle(stream)), "cora_cache_plan")


def rope_table(n_pos, head_dim, theta, device="cuda"):
    """(cos, sin) of pos * theta^(-2 j / head_dim), float32 [n_pos, head_dim / 2, 2], computed in
    64 bits."""
    j = torch.arange(head_dim // 2, dtype=torch.float64, device=device)
    ang = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * theta ** (-2.0 * j / head_dim)
    return torch.stack([torch.cos(ang), torch.sin(ang)], dim=-1).float()


def cache_store(cache: KVCache, layer, x, n_heads, chunk: Chunk, rope=None, q=None, stream=None):
    """Rotate the q and k of x rows [q | k | v] (bf16 or float32, [rows, (n_heads + 2 n_kv_heads)
    head_dim], rows may be strided) and write K and V into the pages (cora_cache_store).  Returns q
    [rows, n_heads, head_dim] bf16; rows that the chunk does not use keep what q held."""
    hd, Hkv = cache.head_dim, cache.n_kv_heads
    width = (n_heads + 2 * Hkv) * hd
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"x: expected a torch.Tensor, got {type(x).__name__}")
    if x.dtype not in (torch.float32,) + _BF16_BITS:
        raise TypeError(f"x: dtype {x.dtype}, expected bfloat16 or float32")
    if not x.is_cuda:
        raise ValueError(f"x: must be a GPU tensor (got device {x.device})")
    if x.dim() != 2 or x.shape[0] < chunk.rows or x.shape[1] != width or x.stride(1) != 1:
        raise ValueError(f"x: shape {tuple(x.shape)} strides {x.stride()}, the call needs "
                         f"[{chunk.rows}, {width}] with rows of stride 1")
    ld = x.stride(0) if x.shape[0] > 1 else width
    if rope is not None:
        check_device_tensor(rope, "rope", (torch.float32,))
        if rope.dim() != 3 or rope.shape[1:] != (hd // 2, 2):
            raise ValueError(f"rope: shape {tuple(rope.shape)}, expected [n_pos, {hd // 2}, 2]")
    if q is None:
        q = torch.empty((chunk.rows, n_heads, hd), dtype=torch.bfloat16, device=x.device)
    check_device_tensor(q, "q", _BF16_BITS, chunk.rows * n_heads * hd)
    _same_device(cache.k, x=x, rope=rope, q=q)
    ca, ch = cache.c(), chunk.c(cache)
    with torch.cuda.device(x.device):
        check(_lib.load().cora_cache_store(ctypes.byref(ca), layer, ptr(x), int(x.dtype == torch.float32),
                                            ld, n_heads, ctypes.byref(ch), chunk.batch, ptr(rope),
                                            0 if rope is None else rope.shape[0], ptr(q),
                                            stream_handle(stream)), "cora_cache_store")
    return q


def cache_attention_workspace(cache: KVCache, n_heads, chunk: Chunk, max_count, max_len):
    """Bytes of workspace that cache_attention needs for these sizes."""
    n = ctypes.c_size_t(0)
    most = cache.max_pages * cache.page_size
    with torch.cuda.device(cache.k.device):
        check(_lib.load().cora_cache_attention_workspace(n_heads, cache.n_kv_heads, cache.head_dim,
                                                          cache.batch, chunk.rows, max_count,
                                                          min(max_len, most) if max_len > 0 else most,
                                                          ctypes.byref(n)),
              "cora_cache_attention_workspace")
    return n.value


def cache_attention(cache: KVCache, layer, q, chunk: Chunk, max_count=0, max_len=0, causal=False,
                    scale=None, out=None, workspace=None, stream=None):
    """Attention of the chunk's rows q [rows, n_heads, head_dim] bf16 over their requests' pages
    (cora_cache_attention).  max_count and max_len: most rows of a request and longest cached
    length to expect (0: the capacities); they choose how the work is split.  workspace: a uint8
    tensor of cache_attention_workspace bytes; by default torch's allocator provides one for the
    call.  Returns out (q's shape); rows that the chunk does not use keep what out held."""
    check_device_tensor(q, "q", _BF16_BITS)
    if q.dim() != 3 or q.shape[0] < chunk.rows or q.shape[2] != cache.head_dim:
        raise ValueError(f"q: shape {tuple(q.shape)}, expected [{chunk.rows}, n_heads, {cache.head_dim}]")
    n_heads = q.shape[1]
    if out is None:
        out = torch.empty_like(q)
    check_device_tensor(out, "out", _BF16_BITS, chunk.rows * n_heads * cache.head_dim)
    _same_device(cache.k, q=q, out=out, workspace=workspace)
    if workspace is None:
        n = cache_attention_workspace(cache, n_heads, chunk, max_count, max_len)
        if n:
            workspace = torch.empty(n, dtype=torch.uint8, device=q.device)
    else:
        check_device_tensor(workspace, "workspace", (torch.uint8,))
    ca, pg, ch = cache.c(), cache.pages(), chunk.c(cache)
    with torch.cuda.device(q.device):
        s = stream_handle(stream)
        check(_lib.load().cora_cache_attention(ctypes.byref(ca), layer, ctypes.byref(pg), ctypes.byref(ch),
                                                ptr(q), n_heads, max_count, max_len, int(bool(causal)),
                                                cache.head_dim ** -0.5 if scale is None else scale,
                                                ptr(out), ptr(workspace),
                                                0 if workspace is None else workspace.numel(), s),
              "cora_cache_attention")
        if workspace is not None and stream is not None:
            workspace.record_stream(stream)
    return out
