"""Host-side checks of the binding of include/maestro_layers.h, without a GPU: the kernels index every array by the sizes a call
passes, so the binding checks each tensor against them before the call. CPU tensors stand in for device tensors and a
recording stub for the library, so nothing is ever launched."""
import pytest
import torch

import paper_2606_12950_amd as M
from paper_2606_12950_amd import _layers, _native, _train

BF16, F32, I8, U8, I64 = torch.bfloat16, torch.float32, torch.int8, torch.uint8, torch.int64


class _Lib:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *args: 64
        return lambda *args: self.calls.append((name, args)) or 0


class _Tensors:
    """The native module, taking part in nothing."""

    def __getattr__(self, name):
        if name == "empties":
            return lambda like, *specs: tuple(torch.empty(s[0], dtype=(F32, torch.int32, like.dtype)[s[1]]) for s in specs)
        return lambda *args: None


@pytest.fixture
def stub(monkeypatch):
    lib = _Lib()

    def dev(t, name, dtype):         # the real check minus the device test
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t

    def matrix(t, name, *dtypes):
        if t.dtype not in dtypes:
            raise TypeError(f"{name} must be one of {dtypes}")
        if t.dim() != 2 or not t.is_contiguous():
            raise ValueError(name)
        return t.shape
    for m in (_native, _train, _layers):
        monkeypatch.setattr(m, "_lib", lib)
        monkeypatch.setattr(m, "_dev", dev)
        monkeypatch.setattr(m, "_stream", lambda s: None)
    monkeypatch.setattr(_train, "_tensors", _Tensors())
    monkeypatch.setattr(_layers, "_tensors", _Tensors())
    monkeypatch.setattr(_layers, "_matrix", matrix)
    monkeypatch.setattr(_layers, "_here", lambda: -1)
    monkeypatch.setattr(_layers, "_raw_stream", lambda device: 0)
    return lib


def e(*shape, dtype=F32):
    return torch.zeros(shape, dtype=dtype)


def refused(stub, call, **bad):
    stub.calls.clear()
    with pytest.raises((ValueError, TypeError)):
        call(**bad)
    assert not stub.calls


def test_layer_grouped(stub):
    ok = dict(x=e(5, 32, dtype=BF16), weight=e(3, 16, 32, dtype=BF16), bias=e(3, 16), offsets=e(4, dtype=I64))
    assert M.layer_grouped(**ok).shape == (5, 16)
    name, args = stub.calls[0]
    assert name == "maestro_layer_grouped" and args[:5] == (5, 3, 32, 16, 1) and args[9] == 1
    for bad in (dict(x=e(5, 16, dtype=BF16)), dict(x=e(5, 32)), dict(weight=e(16, 32, dtype=BF16)), dict(bias=e(16)), dict(bias=e(3, 16, dtype=BF16)),
                dict(offsets=e(3, dtype=I64)), dict(offsets=e(4, dtype=torch.int32)), dict(out=e(5, 16)), dict(out=e(4, 16, dtype=BF16)),
                dict(x=e(32, 5, dtype=BF16).t()), dict(weight=e(3, 16, 32, dtype=torch.float16)), dict(weight=None)):
        refused(stub, M.layer_grouped, **{**ok, **bad})


def test_layer_grouped_grad(stub):
    ok = dict(x=e(5, 32), weight=e(3, 16, 32), g_z=e(5, 16), offsets=e(4, dtype=I64))
    got = M.layer_grouped_grad(**ok)
    assert got.x.shape == (5, 32) and got.weight.shape == (3, 16, 32) and got.bias.shape == (3, 16)
    assert M.layer_grouped_grad(**ok, want_x=False).x is None
    assert stub.calls[0][1][-2] == 64                   # the workspace it asked for
    out = M.LayerGrad(e(5, 32), e(3, 16, 32), e(3, 16))
    M.layer_grouped_grad(**ok, out=out)
    for bad in (dict(g_z=e(4, 16)), dict(g_z=e(5, 16, dtype=BF16)), dict(out=out._replace(x=None)), dict(out=out, want_x=False),
                dict(out=out._replace(weight=e(16, 32))), dict(out=out._replace(bias=e(3, 17))), dict(workspace=e(64)),
                dict(out=out._replace(x=e(6, 32)))):
        refused(stub, M.layer_grouped_grad, **{**ok, **bad})


def test_quantize_rows(stub):
    got = M.quantize_rows(e(5, 32, dtype=BF16))
    assert got.codes.dtype == I8 and got.codes.shape == (5, 32) and got.scale.shape == (5,)
    for bad in (dict(x=e(5, 32, dtype=I8)), dict(x=e(32)), dict(x=e(5, 32), out=M.Quantized(e(5, 32, dtype=U8), e(5))),
                dict(x=e(5, 32), out=M.Quantized(e(5, 32, dtype=I8), e(4)))):
        refused(stub, M.quantize_rows, **bad)


def test_layer_int8(stub):
    ok = dict(x=M.Quantized(e(5, 32, dtype=I8), e(5)), weight=M.Quantized(e(16, 32, dtype=I8), e(16)), bias=e(16))
    assert M.layer_int8(**ok).dtype == BF16 and M.layer_int8(**ok, dtype=F32).dtype == F32
    for bad in (dict(dtype=torch.float16), dict(bias=e(17)), dict(x=M.Quantized(e(5, 32, dtype=I8), e(6))),
                dict(x=M.Quantized(e(5, 16, dtype=I8), e(5))), dict(weight=M.Quantized(e(16, 32, dtype=I8), e(5))),
                dict(weight=M.Quantized(e(16, 32, dtype=U8), e(16))), dict(out=e(5, 16)), dict(dtype=F32, out=e(5, 17))):
        refused(stub, M.layer_int8, **{**ok, **bad})


def test_pack_and_unpack(stub):
    for rectified, dtype in ((False, I8), (True, U8)):
        p = M.pack_activations(e(5, 48, dtype=BF16), rectified=rectified)
        assert p.codes.dtype == dtype and p.exponents.shape == (5, 2) and p.exponents.dtype == U8
        assert M.unpack_activations(p).dtype == BF16
    for bad in (dict(out=M.Packed(e(5, 48, dtype=U8), e(5, 2, dtype=U8))), dict(out=M.Packed(e(5, 48, dtype=I8), e(5, 1, dtype=U8))),
                dict(out=M.Packed(e(4, 48, dtype=I8), e(4, 2, dtype=U8)))):
        refused(stub, M.pack_activations, x=e(5, 48), **bad)
    for bad in (dict(dtype=torch.float16), dict(out=e(5, 48)), dict(dtype=F32, out=e(5, 47)), dict(packed=M.Packed(p.codes, e(5, 3, dtype=U8))),
                dict(packed=M.Packed(e(5, 48), p.exponents))):
        refused(stub, M.unpack_activations, **{"packed": p, **bad})


def test_layer_grad_packed(stub):
    ok = dict(packed=M.Packed(e(5, 48, dtype=U8), e(5, 2, dtype=U8)), weight=e(16, 48, dtype=BF16), g_z=e(5, 16, dtype=BF16))
    got = M.layer_grad_packed(**ok, relu_input=True)
    assert got.x.dtype == BF16 and got.weight.shape == (16, 48) and got.bias.shape == (16,)
    signed = M.Packed(e(5, 48, dtype=I8), e(5, 2, dtype=U8))
    for bad in (dict(packed=signed, relu_input=True), dict(weight=e(16, 32, dtype=BF16)), dict(g_z=e(5, 16)), dict(g_z=e(5, 17, dtype=BF16)),
                dict(weight=e(16, 48, dtype=torch.float16)), dict(weight=None), dict(out=M.LayerGrad(e(5, 48), e(16, 48), e(16)))):
        refused(stub, M.layer_grad_packed, **{**ok, **bad})


def test_another_device_is_refused(stub, monkeypatch):
    monkeypatch.setattr(_layers, "_here", lambda: 0)
    for call in (lambda: M.layer_grouped(e(5, 32), e(3, 16, 32), e(3, 16), e(4, dtype=I64)), lambda: M.quantize_rows(e(5, 32)),
                 lambda: M.layer_grouped_grad(e(5, 32), e(3, 16, 32), e(5, 16), e(4, dtype=I64)), lambda: M.pack_activations(e(5, 32)),
                 lambda: M.unpack_activations(M.Packed(e(5, 32, dtype=I8), e(5, 1, dtype=U8))),
                 lambda: M.layer_int8(M.Quantized(e(5, 32, dtype=I8), e(5)), M.Quantized(e(16, 32, dtype=I8), e(16)), e(16)),
                 lambda: M.layer_grad_packed(M.Packed(e(5, 32, dtype=I8), e(5, 1, dtype=U8)), e(16, 32), e(5, 16))):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert not stub.calls


def test_cpu_tensors_are_refused():
    """By the real checks, the native module's among them."""
    for call in (lambda: M.layer_grouped(e(5, 32), e(3, 16, 32), e(3, 16), e(4, dtype=I64)), lambda: M.quantize_rows(e(5, 32)),
                 lambda: M.pack_activations(e(5, 32)), lambda: M.unpack_activations(M.Packed(e(5, 32, dtype=I8), e(5, 1, dtype=U8))),
                 lambda: M.layer_grouped_grad(e(5, 32), e(3, 16, 32), e(5, 16), e(4, dtype=I64)),
                 lambda: M.layer_int8(M.Quantized(e(5, 32, dtype=I8), e(5)), M.Quantized(e(16, 32, dtype=I8), e(16)), e(16)),
                 lambda: M.layer_grad_packed(M.Packed(e(5, 32, dtype=I8), e(5, 1, dtype=U8)), e(16, 32), e(5, 16)),
                 lambda: M.quantize_rows(None), lambda: M.pack_activations(3)):
        with pytest.raises((TypeError, ValueError, RuntimeError, AssertionError)):
            call()
