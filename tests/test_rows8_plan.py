"""The 8-bit products' plans, on the host: the shapes of the GPU tests reach every kernel that a plan can pick, and the layers'
shapes every way that split sums go on."""
import ctypes
import os
import re

import pytest

from paper_2608_11235_amd import _lib
from tests.test_gpu_rows8_plans import LAYERS, SHAPES

CUS = 256


class Plan(ctypes.Structure):
    _fields_ = [("few", ctypes.c_bool)] + [(n, ctypes.c_int) for n in ("cfg", "mb", "nb", "sq", "kw", "grid", "splits")] \
        + [("ws_floats", ctypes.c_size_t)] + [(n, ctypes.c_int) for n in ("rest", "rest_cfg", "rest_grid")]


def plan(M, N, K, wide=False):
    f = _lib.load()._ZN4cora10rows8_planEiiibi
    f.restype, f.argtypes = Plan, [ctypes.c_int] * 3 + [ctypes.c_bool, ctypes.c_int]
    return f(M, N, K, wide, CUS)


FEW = {False: {(1, 1, 1), (1, 1, 2), (1, 1, 3), (1, 2, 1), (2, 1, 1), (2, 1, 2), (2, 2, 1), (4, 1, 1)},
       True: {(1, 1, 1), (1, 1, 2), (1, 2, 1), (2, 1, 1)}}
TILES = {False: set(range(6)), True: {3, 5}}


@pytest.mark.parametrize("wide", [False, True])
def test_shapes_reach_every_kernel(wide):
    plans = [plan(*s, wide) for s in SHAPES]
    few, tiles = [p for p in plans if p.few], [p for p in plans if not p.few]
    assert {(p.mb, p.nb, p.sq) for p in few} == FEW[wide]
    assert {p.splits for p in few} >= {1, 2, 3, 5}
    assert {p.cfg for p in tiles if p.splits == 1} == {p.cfg for p in tiles if p.splits > 1} == TILES[wide]
    assert {p.splits for p in tiles} == {1, 2, 4, 8}
    assert {p.rest_cfg for p in tiles if p.rest} == ({5} if wide else {1, 2, 4, 5})
    for (M, N, K), p in zip(SHAPES, plans):
        assert p.ws_floats == (p.splits * M * (-(-N // 4) * 4) if p.splits > 1 else 0)
        assert not p.rest or (p.splits == 1 and 0 < p.rest < N and (N - p.rest) % 64 == 0)


@pytest.mark.parametrize("wide", [False, True])
def test_no_size_picks_another_kernel(wide):
    for M in (1, 16, 17, 32, 33, 64):
        for N in (1, 16, 500, 8176, 8177, 37888, 200000):
            for K in (1, 512, 513, 4096, 4097, 8192, 8193, 12288, 12289, 18944, 40000):
                p = plan(M, N, K, wide)
                assert (p.mb, p.nb, p.sq) in FEW[wide] if p.few else p.cfg in TILES[wide]
                assert not p.few or p.kw * p.sq * p.splits >= -(-K // 512)


def test_layers_hand_on_every_kind_of_sums():
    """QKV's to the cache's store, the attention output's and the inner rows' to the residual, added there (2, 4 or 8 of them) or
    before (others)."""
    seen = {"qkv": set(), "out": set(), "gate_up": set(), "down": set()}
    for d, heads, kv, ffn, rows in LAYERS:
        f = -(-ffn // 64) * 64
        for name, N, K in (("qkv", (heads + 2 * kv) * 128, d), ("out", d, heads * 128), ("gate_up", 2 * f, d), ("down", d, f)):
            seen[name].add(plan(rows, N, K).splits)
    print(seen)
    assert seen["qkv"] >= {1, 2} and seen["out"] >= {1, 2} and seen["gate_up"] >= {1, 2} and seen["down"] >= {1, 2, 3, 5, 8}
    assert {4, 8} <= seen["qkv"] | seen["out"] | seen["down"]


@pytest.mark.parametrize("macro,wide", [("R8_FEW", False), ("R8_FEW_WIDE", True)])
def test_every_kernel_of_few_rows_is_picked_by_some_size(macro, wide):
    text = open(os.path.join(os.path.dirname(_lib.__file__), "csrc", "rows8.hip")).read()
    line = re.search(rf"^#define {macro}\(X\)(.*)$", text, re.M).group(1)
    assert {tuple(map(int, x)) for x in re.findall(r"X\((\d), (\d), (\d)\)", line)} == FEW[wide]
