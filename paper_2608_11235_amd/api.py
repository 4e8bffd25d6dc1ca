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
        self._device = torch.cuda.current_device()

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
        device = _device_of(cache, chunk)
        if device != self._device:
            raise ValueError(f"cache: on cuda:{device}, the model is on cuda:{self._device}")
        rows, vocab = chunk._rows, self.spec.vocab
        at = _checked(tokens, "tokens", _I32, rows, device)
        if out is None:
            out = _empty((rows, vocab), torch.int16, tokens.device, stream)
        _call(device, "cora_forward_cached", self._h, cache._cache, cache._pages, chunk._chunk, at, max_count,
              max_len, 1 if causal else 0, _checked(out, "out", _BF16_BITS, rows * vocab, device), stream=stream)
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


# ---- sampling and the paged cache ----------------------------------------------------------------
# These calls take microseconds, so their checks test everything in one expression and look for
# the message only when it fails.
_F32, _I32, _U8 = (torch.float32,), (torch.int32,), (torch.uint8,)


def _checked(t, name, dtypes, numel, device):
    """Address of a contiguous tensor of one of dtypes and at least numel elements on GPU `device`."""
    if not (isinstance(t, torch.Tensor) and t.dtype in dtypes and t.get_device() == device
            and t.is_contiguous() and t.numel() >= numel):
        check_device_tensor(t, name, dtypes, numel)
        raise ValueError(f"{name}: on {t.device}, expected cuda:{device}")
    return t.data_ptr()


def _rows_2d(t, name, dtypes):
    """Check a GPU matrix whose rows are contiguous; returns (device, row stride)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dim() != 2:
        raise ValueError(f"{name}: expected two dimensions, [R, V] or [rows, width], got {tuple(t.shape)}")
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: dtype {t.dtype}, expected one of {dtypes}")
    n, width = t.shape
    if n >> 31 or width >> 31:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, sizes must stay below 2^31")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a GPU tensor (got device {t.device})")
    ld, step = t.stride()
    if (width > 1 and step != 1) or (n > 1 and ld < width):
        raise ValueError(f"{name}: strides {t.stride()}, expected rows of stride 1 that do not overlap")
    return t.get_device(), ld if n > 1 else width


def _call(device, func, *args, stream=None):
    """Call the library with `device` current, on the stream given or torch's current one there."""
    f = getattr(_lib.load(), func)
    if stream is None:
        # the address alone: a torch.cuda.Stream made around it costs a microsecond a call
        handle = torch._C._cuda_getCurrentRawStream(device)
    else:
        if stream.device_index != device:
            raise ValueError(f"stream: on cuda:{stream.device_index}, the tensors are on cuda:{device}")
        handle = stream.cuda_stream
    if torch.cuda.current_device() == device:
        status = f(*args, handle)
    else:
        with torch.cuda.device(device):
            status = f(*args, handle)
    if status:
        check(status, func)


def _empty(shape, dtype, device, stream):
    """A tensor for work on `stream`: from that stream's pool, so that nothing pending on another
    one still uses its memory."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _sample_rows(R, device, temperature, u, top_k, top_p, min_p):
    return _lib.SampleRows(
        _checked(temperature, "temperature", _F32, R, device),
        None if top_k is None else _checked(top_k, "top_k", _I32, R, device),
        None if top_p is None else _checked(top_p, "top_p", _F32, R, device),
        None if min_p is None else _checked(min_p, "min_p", _F32, R, device),
        _checked(u, "u", _F32, R, device))


def vocab_sample(logits, mask_id, temperature, u, top_k=None, top_p=None, min_p=None, token=None,
                 conf=None, stream=None):
    """A token per row of the bf16 logits [R, V] and its confidence (cora_vocab_sample).

    temperature, u, top_p, min_p float32 [R], top_k int32 [R]; top_k, top_p and min_p may be None.
    Rows may be strided (logits.stride(1) == 1); mask_id -1 leaves no id out.  Returns
    (token int32 [R], conf float32 [R])."""
    device, ld = _rows_2d(logits, "logits", _BF16_BITS)
    R, V = logits.shape
    rows = _sample_rows(R, device, temperature, u, top_k, top_p, min_p)
    if token is None:
        token = _empty(R, torch.int32, logits.device, stream)
    if conf is None:
        conf = _empty(R, torch.float32, logits.device, stream)
    _call(device, "cora_vocab_sample", logits.data_ptr(), R, V, ld, mask_id, ctypes.byref(rows),
          _checked(token, "token", _I32, R, device), _checked(conf, "conf", _F32, R, device),
          stream=stream)
    return token, conf


def vocab_gate_sampled(logits, n_rows, row_begin, V, mask_id, state: DecodeState, k_transfer,
                       sched: Sched, gate: Gate, temperature, u, top_k=None, top_p=None, min_p=None,
                       stream=None):
    """vocab_gate with each row's token drawn as by vocab_sample (cora_vocab_gate_sampled)."""
    R = state.B * n_rows
    check_device_tensor(logits, "logits", _BF16_BITS, R * V)
    device = logits.get_device()
    _checked(state.top1, "state.top1", _I32, R, device)
    _checked(state.conf, "state.conf", _F32, R, device)
    rows = _sample_rows(R, device, temperature, u, top_k, top_p, min_p)
    st, sc, gt = state.c(), sched.c(), gate.c()
    _call(device, "cora_vocab_gate_sampled", logits.data_ptr(), n_rows, row_begin, V, mask_id,
          ctypes.byref(st), k_transfer, ctypes.byref(sc), ctypes.byref(gt), ctypes.byref(rows),
          stream=stream)


def _fixed(*names):
    """Read-only attributes: the C structs hold these tensors' addresses."""
    def add(cls):
        for name in names:
            setattr(cls, name, property(lambda self, key="_" + name: getattr(self, key)))
        return cls
    return add


@_fixed("k", "v", "table", "len", "free", "n_free", "n_layers", "n_pages", "n_kv_heads", "head_dim",
        "page_size", "batch", "max_pages")
class KVCache:
    """Paged K and V of n_layers layers and the pages that up to `batch` requests hold of them
    (cora_cache and cora_pages in include/cora.h).  Starts empty, all pages free.  Its tensors are
    its own for good (written in place, never replaced)."""

    def __init__(self, n_layers, n_pages, n_kv_heads, head_dim, page_size, batch, max_pages,
                 device="cuda"):
        self._n_layers, self._n_pages, self._n_kv_heads = n_layers, n_pages, n_kv_heads
        self._head_dim, self._page_size, self._batch, self._max_pages = head_dim, page_size, batch, max_pages
        shape = (n_layers, n_pages, n_kv_heads, page_size * head_dim)
        i32 = torch.int32
        self._k = torch.empty(shape, dtype=torch.bfloat16, device=device)
        self._v = torch.empty(shape, dtype=torch.bfloat16, device=device)
        self._table = torch.full((batch, max_pages), -1, dtype=i32, device=device)
        self._len = torch.zeros(batch, dtype=i32, device=device)
        self._free = torch.arange(n_pages - 1, -1, -1, dtype=i32, device=device)
        self._n_free = torch.full((1,), n_pages, dtype=i32, device=device)
        self._device = self._k.get_device()
        self._workspaces = {}  # bytes that cache_attention needs, by its sizes
        self._cache = ctypes.byref(_lib.Cache(self._k.data_ptr(), self._v.data_ptr(), n_layers, n_pages,
                                              n_kv_heads, page_size, head_dim))
        self._pages = ctypes.byref(_lib.Pages(self._table.data_ptr(), self._len.data_ptr(),
                                              self._free.data_ptr(), self._n_free.data_ptr(), batch,
                                              max_pages, n_pages, page_size))


@_fixed("start", "count", "cu", "positions", "slots", "status", "batch", "rows")
class Chunk:
    """The rows of one pass: positions [start, start + count) of each request, up to `rows` in all
    (cora_chunk).  The caller writes start and count in place; cache_plan writes the rest."""

    def __init__(self, batch, rows, device="cuda"):
        i32 = torch.int32
        self._batch, self._rows = batch, rows
        self._start = torch.zeros(batch, dtype=i32, device=device)
        self._count = torch.zeros(batch, dtype=i32, device=device)
        self._cu = torch.zeros(batch + 1, dtype=i32, device=device)
        self._positions = torch.full((rows,), -1, dtype=i32, device=device)
        self._slots = torch.full((rows,), -1, dtype=i32, device=device)
        self._status = torch.zeros(batch, dtype=i32, device=device)
        self._device = self._start.get_device()
        # rows = 0: torch gives no address for an empty tensor, the library asks for one
        self._chunk = ctypes.byref(_lib.ChunkRows(
            self._start.data_ptr(), self._count.data_ptr(), self._cu.data_ptr(),
            self._positions.data_ptr() or self._cu.data_ptr(), self._slots.data_ptr() or self._cu.data_ptr(),
            self._status.data_ptr(), rows))


def _device_of(cache, chunk):
    if cache._device < 0:
        raise ValueError("cache: must be on a GPU")
    if chunk._device != cache._device:
        raise ValueError(f"chunk: not on the cache's GPU (cuda:{cache._device})")
    if chunk._batch != cache._batch:
        raise ValueError(f"chunk: {chunk._batch} requests, the cache has {cache._batch}")
    return cache._device


def cache_plan(cache: KVCache, chunk: Chunk, reset=False, stream=None):
    """Pages for the chunk and its rows' positions and slots (cora_cache_plan)."""
    _call(_device_of(cache, chunk), "cora_cache_plan", cache._pages, chunk._chunk, 1 if reset else 0,
          stream=stream)


def rope_table(n_pos, head_dim, theta, device="cuda"):
    """(cos, sin) of pos * theta^(-2 j / head_dim), float32 [n_pos, head_dim / 2, 2], computed in
    64 bits."""
    j = torch.arange(head_dim // 2, dtype=torch.float64, device=device)
    ang = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * theta ** (-2.0 * j / head_dim)
    return torch.stack([torch.cos(ang), torch.sin(ang)], dim=-1).float()


_STORED = (torch.float32,) + _BF16_BITS


def cache_store(cache: KVCache, layer, x, n_heads, chunk: Chunk, rope=None, q=None, stream=None):
    """Rotate the q and k of x rows [q | k | v] (bf16 or float32, [rows, (n_heads + 2 n_kv_heads)
    head_dim], rows may be strided) and write K and V into the pages (cora_cache_store).  Returns q
    [rows, n_heads, head_dim] bf16; rows that the chunk does not use keep what q held."""
    device = _device_of(cache, chunk)
    hd, rows = cache._head_dim, chunk._rows
    width = (n_heads + 2 * cache._n_kv_heads) * hd
    xdev, ld = _rows_2d(x, "x", _STORED)
    if x.shape[0] < rows or x.shape[1] != width or xdev != device:
        raise ValueError(f"x: shape {tuple(x.shape)} on {x.device}, the call needs [{rows}, {width}] on "
                         f"cuda:{device}")
    n_pos, angles = 0, None
    if rope is not None:
        angles = _checked(rope, "rope", _F32, 0, device)
        if rope.dim() != 3 or rope.shape[0] < 1 or rope.shape[1:] != (hd // 2, 2):
            raise ValueError(f"rope: shape {tuple(rope.shape)}, expected [n_pos, {hd // 2}, 2]")
        n_pos = rope.shape[0]
    if q is None:
        q = _empty((rows, n_heads, hd), torch.bfloat16, x.device, stream)
    _call(device, "cora_cache_store", cache._cache, layer, x.data_ptr(), 1 if x.dtype is torch.float32 else 0,
          ld, n_heads, chunk._chunk, chunk._batch, angles, n_pos,
          _checked(q, "q", _BF16_BITS, rows * n_heads * hd, device), stream=stream)
    return q


def cache_attention_workspace(cache: KVCache, n_heads, chunk: Chunk, max_count=0, max_len=0):
    """Bytes of workspace that cache_attention needs for these sizes."""
    n = ctypes.c_size_t(0)
    most = cache._max_pages * cache._page_size
    with torch.cuda.device(cache._device):
        check(_lib.load().cora_cache_attention_workspace(
            n_heads, cache._n_kv_heads, cache._head_dim, cache._batch, chunk._rows, max_count,
            min(max_len, most) if max_len > 0 else most, ctypes.byref(n)), "cora_cache_attention_workspace")
    return n.value


def cache_attention(cache: KVCache, layer, q, chunk: Chunk, max_count=0, max_len=0, causal=False,
                    scale=None, out=None, workspace=None, stream=None):
    """Attention of the chunk's rows q [rows, n_heads, head_dim] bf16 over their requests' pages
    (cora_cache_attention).  max_count and max_len: most rows of a request and longest cached
    length to expect (0: the capacities); they choose how the work is split.  workspace: a uint8
    tensor of cache_attention_workspace bytes; by default torch's allocator provides one for the
    call.  Returns out (q's shape); rows that the chunk does not use keep what out held."""
    device = _device_of(cache, chunk)
    rows, hd = chunk._rows, cache._head_dim
    at = _checked(q, "q", _BF16_BITS, 0, device)
    if q.dim() != 3 or q.shape[0] < rows or q.shape[2] != hd:
        raise ValueError(f"q: shape {tuple(q.shape)}, expected [{rows}, n_heads, {hd}]")
    n_heads = q.shape[1]
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    if workspace is None:
        key = (n_heads, rows, max_count, max_len)
        n = cache._workspaces.get(key)
        if n is None:
            if len(cache._workspaces) >= 256:  # a max_len that grows with every call
                cache._workspaces.clear()
            n = cache._workspaces[key] = cache_attention_workspace(cache, n_heads, chunk, max_count, max_len)
        if n:
            workspace = _empty(n, torch.uint8, q.device, stream)
    _call(device, "cora_cache_attention", cache._cache, layer, cache._pages, chunk._chunk, at, n_heads,
          max_count, max_len, 1 if causal else 0, hd ** -0.5 if scale is None else scale,
          _checked(out, "out", _BF16_BITS, rows * n_heads * hd, device),
          None if workspace is None else _checked(workspace, "workspace", _U8, 0, device),
          0 if workspace is None else workspace.numel(), stream=stream)
    return out
