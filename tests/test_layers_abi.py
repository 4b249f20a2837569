"""The C-ABI of include/maestro_layers.h: the library exports what it declares, and every refusal comes from the host before
anything is launched (no GPU needed: none of these calls reaches a kernel)."""
import ctypes
import os
import re

import pytest

from paper_2606_12950_amd import _layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16 = 0, 1

_buf = (ctypes.c_double * 64)()
_at = ctypes.addressof(_buf) + (-ctypes.addressof(_buf) % 16)
A = ctypes.c_void_p(_at)             # 16-byte aligned, never dereferenced
OFF8, OFF4, OFF2, OFF1 = (ctypes.c_void_p(_at + o) for o in (8, 4, 2, 1))


@pytest.fixture(scope="module")
def lib():
    return _layers.load()


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "maestro_layers.h")).read()
    names = sorted(set(re.findall(r"MAESTRO_API\s+[\w\s\*]+?\b(maestro_\w+)\s*\(", text)))
    assert names == sorted(_layers.EXPORTS)
    for n in names:
        assert hasattr(lib, n), n
    assert f"MAESTRO_MAX_LAYER_GROUPS {_layers.MAX_LAYER_GROUPS}\n" in text


WIDTHS = [(dict(i=8), UNSUPPORTED), (dict(o=24), UNSUPPORTED), (dict(i=16400), UNSUPPORTED), (dict(o=16400), UNSUPPORTED),
          (dict(i=0), INVALID), (dict(o=-16), INVALID), (dict(dtype=2), INVALID), (dict(n=-1), INVALID), (dict(n=(1 << 40) + 1), INVALID)]


def _grouped(lib, n=4, g=3, i=32, o=16, dtype=BF16, x=A, w=A, b=A, off=A, y=A):
    return lib.maestro_layer_grouped(n, g, i, o, dtype, x, w, b, off, 1, y, None)


@pytest.mark.parametrize("bad, status", [*WIDTHS, (dict(g=0), INVALID), (dict(g=-1), INVALID), (dict(g=257), UNSUPPORTED), (dict(x=None), INVALID),
                                         (dict(w=None), INVALID), (dict(b=None), INVALID), (dict(off=None), INVALID),
                                         (dict(y=None), INVALID), (dict(x=OFF8), INVALID), (dict(w=OFF8), INVALID),
                                         (dict(b=OFF8), INVALID), (dict(off=OFF4), INVALID), (dict(y=OFF8), INVALID)])
def test_grouped_refuses(lib, bad, status):
    assert _grouped(lib, **bad) == status


def test_grouped_without_rows(lib):
    assert _grouped(lib, n=0, x=None, y=None) == OK
    assert _grouped(lib, n=0, x=None, y=None, off=None) == INVALID


def _grouped_grad(lib, n=20000, g=3, i=32, o=16, dtype=BF16, x=A, w=A, gz=A, off=A, gx=A, gw=A, gb=A, ws=A, size=1 << 40):
    return lib.maestro_layer_grouped_grad(n, g, i, o, dtype, x, w, gz, off, 0, gx, gw, gb, ws, size, None)


@pytest.mark.parametrize("bad, status", [*WIDTHS, (dict(g=0), INVALID), (dict(g=257), UNSUPPORTED), (dict(x=None), INVALID), (dict(w=None), INVALID),
                                         (dict(gz=None), INVALID), (dict(off=None), INVALID), (dict(gw=None), INVALID),
                                         (dict(gb=None), INVALID), (dict(gx=OFF8), INVALID), (dict(gz=OFF8), INVALID),
                                         (dict(off=OFF4), INVALID), (dict(gw=OFF4), INVALID), (dict(gb=OFF8), INVALID),
                                         (dict(ws=None), INVALID), (dict(ws=OFF8), INVALID), (dict(size=0), WORKSPACE)])
def test_grouped_grad_refuses(lib, bad, status):
    assert _grouped_grad(lib, **bad) == status


def test_grouped_grad_workspace(lib):
    ws = lib.maestro_layer_grouped_grad_workspace
    for dtype in (F32, BF16):
        for n in (20000, 262139, 1 << 30):
            need = ws(n, 3, 32, 16, dtype)
            assert need >= 4 * 33 * 16 and need % 4 == 0
            assert _grouped_grad(lib, n=n, dtype=dtype, size=need - 1) == WORKSPACE
        assert ws(0, 3, 32, 16, dtype) == ws(100, 3, 32, 16, dtype) == 0          # no group has more than one share
    assert ws((1 << 31) - (1 << 16) + 1, 3, 32, 16, BF16) == 0
    assert _grouped(lib, n=(1 << 31) - (1 << 16) + 1) == _grouped_grad(lib, n=(1 << 31) - (1 << 16) + 1) == UNSUPPORTED
    assert _grouped(lib, n=1 << 30, i=16384) == UNSUPPORTED
    assert ws(4, 0, 32, 16, BF16) == ws(4, 257, 32, 16, BF16) == ws(4, 3, 24, 16, BF16) == ws(-1, 3, 32, 16, BF16) == 0


def _quantize(lib, n=4, i=32, dtype=BF16, x=A, codes=A, scale=A):
    return lib.maestro_quantize_rows(n, i, dtype, x, codes, scale, None)


@pytest.mark.parametrize("bad, status", [(b, s) for b, s in WIDTHS if "o" not in b] +
                         [(dict(x=None), INVALID), (dict(codes=None), INVALID), (dict(scale=None), INVALID), (dict(x=OFF8), INVALID),
                          (dict(codes=OFF8), INVALID), (dict(scale=OFF2), INVALID)])
def test_quantize_refuses(lib, bad, status):
    assert _quantize(lib, **bad) == status
    assert _quantize(lib, n=0, x=None, codes=None, scale=None) == OK


def _int8(lib, n=4, i=32, o=16, dtype=BF16, x=A, xs=A, w=A, ws=A, b=A, y=A):
    return lib.maestro_layer_int8(n, i, o, x, xs, w, ws, b, 1, dtype, y, None)


@pytest.mark.parametrize("bad, status", [*WIDTHS, (dict(x=None), INVALID), (dict(xs=None), INVALID), (dict(w=None), INVALID),
                                         (dict(ws=None), INVALID), (dict(b=None), INVALID), (dict(y=None), INVALID),
                                         (dict(x=OFF8), INVALID), (dict(xs=OFF2), INVALID), (dict(w=OFF8), INVALID),
                                         (dict(ws=OFF8), INVALID), (dict(b=OFF8), INVALID), (dict(y=OFF8), INVALID)])
def test_int8_refuses(lib, bad, status):
    assert _int8(lib, **bad) == status
    assert _int8(lib, n=0, x=None, xs=None, y=None) == OK


def _pack(lib, n=4, i=32, dtype=BF16, x=A, codes=A, e=A):
    return lib.maestro_pack_activations(n, i, dtype, x, 1, codes, e, None)


def _unpack(lib, n=4, i=32, dtype=BF16, x=A, codes=A, e=A):
    return lib.maestro_unpack_activations(n, i, dtype, codes, e, 1, x, None)


@pytest.mark.parametrize("call", [_pack, _unpack])
@pytest.mark.parametrize("bad, status", [(b, s) for b, s in WIDTHS if "o" not in b] +
                         [(dict(x=None), INVALID), (dict(codes=None), INVALID), (dict(e=None), INVALID), (dict(x=OFF8), INVALID),
                          (dict(codes=OFF8), INVALID)])
def test_pack_refuses(lib, call, bad, status):
    assert call(lib, **bad) == status
    assert call(lib, n=0, x=None, codes=None, e=None) == OK


def _packed_grad(lib, n=4, i=32, o=16, dtype=BF16, codes=A, e=A, rectified=1, w=A, gz=A, relu=1, gx=A, gw=A, gb=A, ws=A, size=1 << 50):
    return lib.maestro_layer_grad_packed(n, i, o, dtype, codes, e, rectified, w, gz, relu, gx, gw, gb, ws, size, None)


@pytest.mark.parametrize("bad, status", [*WIDTHS, (dict(codes=None), INVALID), (dict(e=None), INVALID), (dict(w=None), INVALID),
                                         (dict(gz=None), INVALID), (dict(gw=None), INVALID), (dict(gb=None), INVALID),
                                         (dict(codes=OFF8), INVALID), (dict(gx=OFF8), INVALID), (dict(gz=OFF8), INVALID),
                                         (dict(gw=OFF8), INVALID), (dict(gb=OFF4), INVALID), (dict(rectified=0), INVALID)])
def test_packed_grad_refuses(lib, bad, status):
    assert _packed_grad(lib, **bad) == status


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_grad_workspace(lib, dtype):
    for n, i, o in ((70000, 64, 128), (300, 256, 512), (1 << 33, 1024, 64)):
        need = lib.maestro_layer_grad_packed_workspace(n, i, o, dtype)
        if need:
            assert _packed_grad(lib, n=n, i=i, o=o, dtype=dtype, size=need - 1) == WORKSPACE
            assert _packed_grad(lib, n=n, i=i, o=o, dtype=dtype, ws=None) == INVALID
    assert lib.maestro_layer_grad_packed_workspace(4, 24, 16, dtype) == lib.maestro_layer_grad_packed_workspace(-1, 32, 16, dtype) == 0
