"""The sampling and cache entry points refuse malformed calls on the host, before any GPU work
(no GPU needed), and the binding refuses tensors that the library would misread."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import paper_2608_11235_amd as pkg
from paper_2608_11235_amd import api
from tests import cache_ref as ref

FAKE = 1 << 20  # a non-null, aligned address that a refused call never follows
INVALID, UNSUPPORTED = -1, -2


@pytest.fixture(scope="module")
def lib():
    from paper_2608_11235_amd import _lib as L
    if not os.path.exists(L.LIB_PATH):
        pytest.fail("libcora.so is not built (run __graft_entry__.build())")
    return L


def cache(L, **kw):
    base = dict(k=FAKE, v=FAKE, n_layers=2, n_pages=8, n_kv_heads=2, page_size=64, head_dim=128)
    return L.Cache(**{**base, **kw})


def pages(L, **kw):
    base = dict(table=FAKE, len=FAKE, free=FAKE, n_free=FAKE, B=2, max_pages=4, n_pages=8, page_size=64)
    return L.Pages(**{**base, **kw})


def chunk(L, **kw):
    base = dict(start=FAKE, count=FAKE, cu=FAKE, positions=FAKE, slots=FAKE, status=FAKE, rows=16)
    return L.ChunkRows(**{**base, **kw})


def test_struct_layouts_match_the_header(lib, tmp_path):
    from tests.test_abi import ROOT
    import subprocess
    structs = {"cora_sample_rows": lib.SampleRows, "cora_cache": lib.Cache, "cora_pages": lib.Pages,
               "cora_chunk": lib.ChunkRows}
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "cora.h"', "int main(void){"]
    for c, py in structs.items():
        src.append(f'printf("{c} size %zu\\n", sizeof({c}));')
        src += [f'printf("{c} {f} %zu\\n", offsetof({c}, {f}));' for f, _ in py._fields_]
    (tmp_path / "l.c").write_text("\n".join(src + ["return 0;}"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")])
    got = {tuple(x.split()[:2]): int(x.split()[2])
           for x in subprocess.check_output([str(tmp_path / "l")], text=True).splitlines()}
    for c, py in structs.items():
        assert got[(c, "size")] == ctypes.sizeof(py)
        for f, _ in py._fields_:
            assert got[(c, f)] == getattr(py, f).offset, (c, f)


@pytest.mark.parametrize("R,V,ld,mask,status", [
    (-1, 10, 10, 0, INVALID), (2, 0, 10, -1, INVALID), (2, 10, 9, 0, INVALID), (2, 10, 10, 10, INVALID),
    (2, 10, 10, -2, INVALID), (2, (1 << 30) + 1, 1 << 31, 0, UNSUPPORTED), (0, 10, 10, 0, 0)])
def test_vocab_sample(lib, R, V, ld, mask, status):
    rows = lib.SampleRows(temperature=FAKE, u=FAKE)
    assert lib.load().cora_vocab_sample(FAKE, R, V, ld, mask, ctypes.byref(rows), FAKE, FAKE, None) == status


def test_vocab_sample_null_arrays(lib):
    f = lib.load().cora_vocab_sample
    ok = lib.SampleRows(temperature=FAKE, u=FAKE)
    assert f(None, 2, 10, 10, 0, ctypes.byref(ok), FAKE, FAKE, None) == INVALID
    assert f(FAKE, 2, 10, 10, 0, ctypes.byref(ok), None, FAKE, None) == INVALID
    assert f(FAKE, 2, 10, 10, 0, ctypes.byref(ok), FAKE, None, None) == INVALID
    assert f(FAKE, 2, 10, 10, 0, None, FAKE, FAKE, None) == INVALID
    for bad in (lib.SampleRows(temperature=FAKE), lib.SampleRows(u=FAKE)):
        assert f(FAKE, 2, 10, 10, 0, ctypes.byref(bad), FAKE, FAKE, None) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(table=None), INVALID), (dict(len=None), INVALID), (dict(free=None), INVALID), (dict(n_free=None), INVALID),
    (dict(B=0), INVALID), (dict(max_pages=0), INVALID), (dict(n_pages=0), INVALID), (dict(B=4097), UNSUPPORTED),
    (dict(page_size=48), UNSUPPORTED), (dict(page_size=16), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(max_pages=1 << 25), UNSUPPORTED), (dict(n_pages=1 << 25), UNSUPPORTED)])
def test_plan_pages(lib, kw, status):
    c = chunk(lib)
    assert lib.load().cora_cache_plan(ctypes.byref(pages(lib, **kw)), ctypes.byref(c), 0, None) == status


@pytest.mark.parametrize("kw", [dict(start=None), dict(count=None), dict(cu=None), dict(positions=None),
                                dict(slots=None), dict(status=None), dict(rows=-1), dict(rows=(1 << 28) + 1)])
def test_plan_chunk(lib, kw):
    assert lib.load().cora_cache_plan(ctypes.byref(pages(lib)), ctypes.byref(chunk(lib, **kw)), 0, None) == INVALID
    assert lib.load().cora_cache_plan(None, ctypes.byref(chunk(lib)), 0, None) == INVALID
    assert lib.load().cora_cache_plan(ctypes.byref(pages(lib)), None, 0, None) == INVALID


def store(lib, ca=None, ch=None, layer=0, x=FAKE, f32=0, ld=8 * 128, heads=4, B=2, rope=FAKE, n_pos=10, q=FAKE):
    return lib.load().cora_cache_store(ctypes.byref(ca or cache(lib)), layer, x, f32, ld, heads,
                                       ctypes.byref(ch or chunk(lib)), B, rope, n_pos, q, None)


def test_store(lib):
    assert store(lib, layer=2) == INVALID and store(lib, layer=-1) == INVALID
    assert store(lib, x=None) == INVALID and store(lib, x=FAKE + 8) == INVALID
    assert store(lib, q=FAKE + 2) == INVALID and store(lib, rope=FAKE + 4) == INVALID
    assert store(lib, ld=8 * 128 - 8) == INVALID and store(lib, ld=8 * 128 + 4) == INVALID
    assert store(lib, ld=8 * 128 + 2, f32=1) == INVALID
    assert store(lib, n_pos=0) == INVALID and store(lib, B=0) == INVALID and store(lib, heads=0) == INVALID
    assert store(lib, heads=3) == UNSUPPORTED
    for kw, status in ((dict(k=None), INVALID), (dict(v=FAKE + 8), INVALID), (dict(head_dim=96), UNSUPPORTED),
                       (dict(page_size=100), UNSUPPORTED), (dict(n_pages=1 << 25), UNSUPPORTED),
                       (dict(n_layers=0), INVALID), (dict(n_kv_heads=0), INVALID)):
        assert store(lib, ca=cache(lib, **kw)) == status, kw
    assert store(lib, ch=chunk(lib, slots=None)) == INVALID
    assert store(lib, ch=chunk(lib, rows=1 << 27), heads=32) == UNSUPPORTED


def attend(lib, ca=None, pg=None, ch=None, layer=0, q=FAKE, heads=4, count=0, length=0, causal=0, scale=0.1,
           out=FAKE, ws=FAKE, n=1 << 40):
    return lib.load().cora_cache_attention(ctypes.byref(ca or cache(lib)), layer, ctypes.byref(pg or pages(lib)),
                                           ctypes.byref(ch or chunk(lib)), q, heads, count, length, causal, scale,
                                           out, ws, n, None)


def test_attention(lib):
    assert attend(lib, q=None) == INVALID and attend(lib, out=None) == INVALID
    assert attend(lib, q=FAKE + 8) == INVALID and attend(lib, out=FAKE + 2) == INVALID
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert attend(lib, scale=scale) == INVALID
    assert attend(lib, heads=5) == UNSUPPORTED and attend(lib, layer=2) == INVALID
    assert attend(lib, pg=pages(lib, page_size=32)) == INVALID
    assert attend(lib, pg=pages(lib, n_pages=7)) == INVALID


def test_attention_workspace(lib):
    f, n = lib.load().cora_cache_attention_workspace, ctypes.c_size_t(0)
    assert f(4, 2, 128, 2, 16, 8, 4096, ctypes.byref(n)) == 0
    big = pages(lib, max_pages=64)
    if n.value:
        kw = dict(pg=big, count=8, length=4096)
        assert attend(lib, ws=None, n=0, **kw) == INVALID
        assert attend(lib, n=n.value - 1, **kw) == INVALID
        assert attend(lib, ws=FAKE + 8, n=n.value, **kw) == INVALID
    assert n.value > 0  # 8 rows over 4096 keys are split
    assert f(4, 2, 128, 2, 16, 8, 4096, None) == INVALID
    assert f(4, 2, 96, 2, 16, 8, 4096, ctypes.byref(n)) == UNSUPPORTED
    assert f(4, 3, 128, 2, 16, 8, 4096, ctypes.byref(n)) == UNSUPPORTED
    assert f(4, 2, 128, 0, 16, 8, 4096, ctypes.byref(n)) == INVALID
    assert f(4, 2, 128, 2, 16, 8, 0, ctypes.byref(n)) == INVALID


def test_forward_cached_null(lib):
    assert lib.load().cora_forward_cached(None, None, None, None, None, 0, 0, 0, None, None) == INVALID


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 8), dtype=torch.bfloat16)
    one = torch.ones(2)
    with pytest.raises(ValueError, match="GPU"):
        pkg.vocab_sample(x, 0, one, one)
    with pytest.raises(TypeError, match="logits"):
        pkg.vocab_sample(np.zeros((2, 8)), 0, one, one)
    with pytest.raises(ValueError, match=r"\[R, V\]"):
        pkg.vocab_sample(x[0], 0, one, one)
    ca = api.KVCache(1, 4, 1, 64, 32, 2, 2, device="cpu")
    ch = api.Chunk(2, 8, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        pkg.cache_plan(ca, ch)
    with pytest.raises(ValueError, match="GPU"):
        pkg.cache_store(ca, 0, torch.zeros((8, 192), dtype=torch.bfloat16), 1, ch)
    with pytest.raises(ValueError, match="GPU"):
        pkg.cache_attention(ca, 0, torch.zeros((8, 1, 64), dtype=torch.bfloat16), ch)
    st = api.DecodeState(1, 8, 32, 16, 16, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        pkg.vocab_gate_sampled(torch.zeros((1, 16, 8), dtype=torch.bfloat16), 16, -1, 8, 0, st, -1, api.Sched(16, 4),
                               api.Gate(), one, one)


def test_rope_table_is_rounded_from_64_bits():
    t = pkg.rope_table(70001, 128, 5e5, device="cpu")[-1].double().numpy()
    ang = 70000.0 * 5e5 ** (-2.0 * np.arange(64) / 128)
    assert np.abs(t - np.stack([np.cos(ang), np.sin(ang)], -1)).max() <= 2.0 ** -24


@pytest.mark.parametrize("page,hd", [(32, 64), (64, 128), (256, 128)])
def test_page_order(page, hd):
    """The reference's offsets are a permutation of a page, and 32 keys stay together."""
    for t in ref.offsets(page, hd):
        assert sorted(t.reshape(-1).tolist()) == list(range(page * hd))
        assert (t // (32 * hd) == torch.arange(page)[:, None] // 32).all()


def test_reference_sampler():
    """The reference itself: hand-worked rows."""
    l = np.log([0.5, 0.25, 0.125, 0.125])
    assert [ref.sample_row(l, -1, 1.0, u)[0] for u in (0.0, 0.49, 0.51, 0.74, 0.76, 0.9)] == [0, 0, 1, 1, 2, 3]
    assert ref.sample_row(l, -1, 1.0, 0.9, top_k=2)[0] == 1           # 2/3, 1/3
    assert ref.sample_row(l, -1, 1.0, 0.99, top_p=0.7)[0] == 1
    assert ref.sample_row(l, -1, 1.0, 0.99, min_p=0.3)[0] == 1
    assert ref.sample_row(l, 0, 1.0, 0.49)[0] == 1                    # id 0 left out: 1/2, 1/4, 1/4
    assert abs(ref.sample_row(l, 0, 1.0, 0.49)[1] - 0.5) < 1e-12
    assert ref.sample_row(l, -1, 0.0, 0.99)[0] == 0
    assert ref.sample_row([1.0, 1.0, 1.0], -1, 0.5, 0.67)[0] == 2
    assert ref.sample_row([-np.inf, -np.inf], -1, 1.0, 0.5) == (-1, 0.0)


def test_reference_plan():
    p = ref.Plan(2, 3, 3, 32)
    o = p.step([0, 0], [40, 20], 64)
    assert o["cu"] == [0, 40, 60] and list(o["status"]) == [0, 0] and p.table[0, :2].tolist() == [0, 1]
    assert o["slots"][40] == 64 and o["slots"][60:] == [-1] * 4
    o = p.step([40, 20], [30, 1], 64)                                 # no page left for the first
    assert list(o["status"]) == [-3, 0] and o["cu"] == [0, 0, 1]
    p.step([0, 0], [-1, 0], 64)
    assert p.len.tolist() == [0, 21] and len(p.free) == 2
