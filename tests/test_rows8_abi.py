"""The 8-bit entry points refuse malformed calls on the host, before any GPU work (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_11235_amd as pkg
from tests.test_cache_abi import FAKE, INVALID, UNSUPPORTED, lib  # noqa: F401


def rows8(L, **kw):
    return L.Rows8(**{**dict(data=FAKE, scale=FAKE, rows=4, cols=256), **kw})


def quantize(L, out=None, x=FAKE, f32=0, ld=256):
    return L.load().cora_quantize_rows(x, f32, ld, ctypes.byref(out or rows8(L)), None)


def product(L, a=None, w=None, bias=None, out=FAKE, f32=0, ld=1 << 26, ws=FAKE, n=1 << 40):
    return L.load().cora_rows_product(ctypes.byref(a or rows8(L)), ctypes.byref(w or rows8(L)), bias, out, f32, ld, ws, n, None)


BAD = [(dict(data=None), INVALID), (dict(scale=None), INVALID), (dict(data=FAKE + 8), INVALID),
       (dict(scale=FAKE + 2), INVALID), (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=-1), INVALID),
       (dict(rows=(1 << 27) + 1), UNSUPPORTED), (dict(cols=(1 << 20) + 1), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", BAD)
def test_rows(lib, kw, status):  # noqa: F811
    assert quantize(lib, rows8(lib, **kw)) == status
    assert product(lib, a=rows8(lib, **kw)) == status and product(lib, w=rows8(lib, **kw)) == status


def test_quantize(lib):  # noqa: F811
    assert quantize(lib, x=None) == INVALID and quantize(lib, ld=255) == INVALID
    assert quantize(lib, x=FAKE + 1) == INVALID and quantize(lib, x=FAKE + 2, f32=1) == INVALID
    assert quantize(lib, rows8(lib, rows=1 << 27)) == UNSUPPORTED
    assert quantize(lib, rows8(lib, rows=1 << 20, cols=1 << 20), ld=1 << 20) == UNSUPPORTED
    assert quantize(lib, rows8(lib, rows=(1 << 27) - 15, cols=1), ld=1) == UNSUPPORTED  # 2^23 workgroups of 512 threads
    assert quantize(lib, rows8(lib, rows=0, data=None, scale=None), x=None) == 0
    assert lib.load().cora_quantize_rows(FAKE, 0, 256, None, None) == INVALID


def test_product(lib):  # noqa: F811
    assert product(lib, out=None) == INVALID and product(lib, ld=3) == INVALID
    assert product(lib, out=FAKE + 1) == INVALID and product(lib, out=FAKE + 2, f32=1) == INVALID
    assert product(lib, bias=FAKE + 2) == INVALID
    assert product(lib, w=rows8(lib, cols=128)) == INVALID
    assert product(lib, a=rows8(lib, rows=(1 << 21) + 1)) == UNSUPPORTED
    assert product(lib, w=rows8(lib, rows=(1 << 25) + 1)) == UNSUPPORTED
    assert product(lib, a=rows8(lib, rows=1 << 20), w=rows8(lib, rows=(1 << 20) + 1), ld=1 << 21) == UNSUPPORTED
    assert product(lib, a=rows8(lib, rows=0, data=None, scale=None), out=None) == 0
    assert lib.load().cora_rows_product(None, None, None, FAKE, 0, 4, None, 0, None) == INVALID


def test_sizes(lib):  # noqa: F811
    f, d, s = lib.load().cora_rows_bytes, ctypes.c_size_t(0), ctypes.c_size_t(0)
    for R, K, want in ((0, 1, (0, 0)), (1, 1, (2048, 64)), (16, 128, (2048, 64)), (17, 129, (8192, 128)),
                       (40, 513, (3 * 5 * 2048, 3 * 2 * 64)), (1 << 27, 1 << 20, (1 << 47, 1 << 40))):
        assert f(R, K, ctypes.byref(d), ctypes.byref(s)) == 0 and (d.value, s.value) == want
    assert f(1, 0, ctypes.byref(d), ctypes.byref(s)) == INVALID and f(1, 1, None, ctypes.byref(s)) == INVALID
    g = lib.load().cora_rows_product_workspace
    assert g(32, 4096, 4096, 0, ctypes.byref(d)) == 0
    assert g(32, 4096, 4096, 1, None) == INVALID and g(32, 4096, 0, 0, ctypes.byref(d)) == INVALID
    assert g(32, (1 << 25) + 1, 64, 0, ctypes.byref(d)) == UNSUPPORTED


def test_product_workspace_is_checked(lib):  # noqa: F811
    n = ctypes.c_size_t(0)
    seen = 0
    for M, N, K, f32 in ((32, 4096, 12288, 0), (32, 4096, 12288, 1), (512, 4096, 12288, 0), (300, 256, 4096, 1), (64, 3584, 18944, 0)):
        assert lib.load().cora_rows_product_workspace(M, N, K, f32, ctypes.byref(n)) == 0
        if n.value:
            a, w = rows8(lib, rows=M, cols=K), rows8(lib, rows=N, cols=K)
            assert product(lib, a, w, f32=f32, ws=None) == INVALID and product(lib, a, w, f32=f32, ws=FAKE + 8) == INVALID
            assert product(lib, a, w, f32=f32, n=n.value - 1) == INVALID
            seen += 1
    assert seen >= 3


def test_layout_matches_the_header(lib, tmp_path):  # noqa: F811
    import os
    import subprocess
    from tests.test_abi import ROOT
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "cora.h"\nint main(void){printf("%zu", sizeof(cora_rows8));'
    src += "".join(f'printf(" %zu", offsetof(cora_rows8, {f}));' for f, _ in lib.Rows8._fields_) + "return 0;}"
    (tmp_path / "l.c").write_text(src)
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "l")], text=True).split()]
    assert got == [ctypes.sizeof(lib.Rows8)] + [getattr(lib.Rows8, f).offset for f, _ in lib.Rows8._fields_]


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError, match="GPU"):
        pkg.quantize_rows(torch.zeros((4, 128)))
    with pytest.raises(TypeError, match="x"):
        pkg.quantize_rows(np.zeros((4, 128)))
    with pytest.raises(TypeError, match="dtype"):
        pkg.quantize_rows(torch.zeros((4, 128), dtype=torch.float16))
    a = pkg.Rows8(4, 128, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        pkg.rows8_product(a, a)
    with pytest.raises(ValueError, match="GPU"):
        pkg.rows8_product_workspace(a, a)
    with pytest.raises(AttributeError):
        a.data = None


def test_values_of_fresh_rows_are_zero():
    assert (pkg.Rows8(5, 200, device="cpu").values() == 0).all()
