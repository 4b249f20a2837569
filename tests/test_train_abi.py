"""The training operators' C-ABI: the library exports what include/maestro_train.h declares, and every
refusal comes from the host before anything is launched (no GPU needed: none of these calls reaches a kernel)."""
import ctypes
import math
import os
import re

import pytest

from paper_2606_12950_amd import _train

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16 = 0, 1

_buf = (ctypes.c_double * 64)()
_at = ctypes.addressof(_buf) + (-ctypes.addressof(_buf) % 16)
A = ctypes.c_void_p(_at)             # 16-byte aligned, never dereferenced
OFF8, OFF4, OFF2, OFF1 = (ctypes.c_void_p(_at + o) for o in (8, 4, 2, 1))


@pytest.fixture(scope="module")
def lib():
    return _train.load()


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "maestro_train.h")).read()
    names = sorted(set(re.findall(r"MAESTRO_API\s+[\w\s\*]+?\b(maestro_\w+)\s*\(", text)))
    assert names == sorted(_train.EXPORTS)
    for n in names:
        assert hasattr(lib, n), n
    assert f"MAESTRO_MAX_ALTERNATIVES {_train.MAX_ALTERNATIVES}\n" in text


def _logprobs(lib, n=4, v=10, x=A, stride=10, dtype=F32, token=A, k=2, lp=A, ent=A, ids=A, top=A, stats=A, ws=A,
              ws_bytes=1 << 30):
    return lib.maestro_logprobs(n, v, x, stride, dtype, token, k, lp, ent, ids, top, stats, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(v=0), dict(k=-1), dict(k=17), dict(dtype=2), dict(stride=9),
                                 dict(x=None), dict(x=OFF2), dict(x=OFF1, dtype=BF16), dict(token=None), dict(lp=None),
                                 dict(token=OFF2), dict(lp=OFF2), dict(ent=OFF2), dict(ids=None), dict(top=None),
                                 dict(ids=OFF1), dict(top=OFF2), dict(stats=OFF4), dict(n=1 << 41),
                                 dict(n=1 << 39, stride=1 << 39), dict(stride=1 << 41)])
def test_logprobs_refuses(lib, bad):
    assert _logprobs(lib, **bad) == INVALID


def test_logprobs_nothing_to_do(lib):
    assert _logprobs(lib, n=0, x=None, ids=None, top=None) == OK
    assert _logprobs(lib, token=None, lp=None, ent=None, stats=None, k=0, ids=None, top=None) == OK


def _grad(lib, n=4, v=10, x=A, stride=10, dtype=F32, token=A, stats=A, ent=A, g=A, ge=A, grad=A, grad_stride=10):
    return lib.maestro_logprobs_grad(n, v, x, stride, dtype, token, stats, ent, g, ge, grad, grad_stride, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(v=0), dict(dtype=-1), dict(stride=9), dict(grad_stride=9), dict(x=None),
                                 dict(grad=None), dict(stats=None), dict(stats=OFF4), dict(token=None), dict(g=None),
                                 dict(token=None, g=None, ge=None), dict(ent=None), dict(grad=OFF2), dict(x=OFF2),
                                 dict(g=OFF2), dict(ge=OFF2), dict(ent=OFF2), dict(token=OFF2),
                                 dict(grad_stride=11)])       # in place, but another stride
def test_logprobs_grad_refuses(lib, bad):
    assert _grad(lib, **bad) == INVALID


def test_logprobs_grad_empty(lib):
    assert _grad(lib, n=0, x=None, grad=None, stats=None) == OK


def _layer(lib, n=4, i=32, o=16, dtype=BF16, x=A, w=A, b=A, y=A):
    return lib.maestro_layer(n, i, o, dtype, x, w, b, 1, y, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(i=0), dict(o=-16), dict(dtype=3), dict(x=None), dict(w=None), dict(b=None),
                                 dict(y=None), dict(x=OFF8), dict(w=OFF8), dict(b=OFF8), dict(y=OFF8)])
def test_layer_refuses(lib, bad):
    assert _layer(lib, **bad) == INVALID


@pytest.mark.parametrize("shape", [dict(i=24), dict(o=8), dict(i=16400), dict(o=16400)])
def test_layer_widths(lib, shape):
    assert _layer(lib, **shape) == UNSUPPORTED
    assert _layer_grad(lib, **shape) == UNSUPPORTED


def test_layer_empty(lib):
    assert _layer(lib, n=0, x=None, y=None) == OK


def _layer_grad(lib, n=4, i=32, o=16, dtype=BF16, x=A, w=A, gz=A, gx=A, gw=A, gb=A, ws=A, ws_bytes=1 << 40):
    return lib.maestro_layer_grad(n, i, o, dtype, x, w, gz, 1, gx, gw, gb, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(i=0), dict(o=0), dict(dtype=3), dict(x=None), dict(w=None), dict(gz=None),
                                 dict(gw=None), dict(gb=None), dict(x=OFF8), dict(w=OFF8), dict(gz=OFF8), dict(gx=OFF8),
                                 dict(gw=OFF8), dict(gb=OFF8)])
def test_layer_grad_refuses(lib, bad):
    assert _layer_grad(lib, **bad) == INVALID


def test_layer_grad_workspace(lib):
    need = lib.maestro_layer_grad_workspace(1 << 20, 1024, 1024, BF16)
    if need:
        assert _layer_grad(lib, n=1 << 20, i=1024, o=1024, ws_bytes=need - 1) == WORKSPACE
        assert _layer_grad(lib, n=1 << 20, i=1024, o=1024, ws=None) == INVALID
        assert _layer_grad(lib, n=1 << 20, i=1024, o=1024, ws=OFF8, ws_bytes=need) == INVALID
    assert lib.maestro_layer_grad_workspace(-1, 16, 16, BF16) == 0
    assert lib.maestro_layer_grad_workspace(1, 24, 16, BF16) == 0


def _clip(lib, n=2, ptr=(A, A), out=None, sizes=(3, 0), dtypes=(F32, BF16), max_norm=1.0, norm=A, ws=A, ws_bytes=1 << 20):
    arr = lambda p: None if p is None else (ctypes.c_void_p * n)(*[q.value if q is not None else None for q in p])
    return lib.maestro_clip_gradients(n, arr(ptr), arr(out), (ctypes.c_int64 * n)(*sizes), (ctypes.c_int32 * n)(*dtypes),
                                      max_norm, norm, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(ptr=None), dict(ptr=(None, A)), dict(ptr=(OFF2, A)), dict(ptr=(A, OFF1), sizes=(1, 1)),
                                 dict(out=(None, A)), dict(out=(OFF2, A)), dict(sizes=(-1, 2)), dict(dtypes=(0, 2)),
                                 dict(max_norm=-1.0), dict(max_norm=math.nan), dict(norm=None), dict(norm=OFF2),
                                 dict(max_norm=math.inf, out=(A, A)), dict(ws=None), dict(ws=OFF8)])
def test_clip_refuses(lib, bad):
    assert _clip(lib, **bad) == INVALID


def test_clip_workspace(lib):
    assert _clip(lib, ws_bytes=lib.maestro_clip_gradients_workspace(2) - 1) == WORKSPACE
    assert lib.maestro_clip_gradients(-1, None, None, None, None, 1.0, A, A, 1 << 20, None) == INVALID


def test_clip_tensors_past_half_a_tebibyte(lib):
    assert _clip(lib, sizes=((1 << 37) + 1, 0)) == INVALID and _clip(lib, dtypes=(BF16, BF16), sizes=((1 << 38) + 1, 0)) == INVALID
