"""Thin ctypes binding of the layers by role, in 8-bit integers and from 8-bit checkpoints (include/maestro_layers.h).

Argument marshalling only, in the manner of ``_train``: the tensors are checked, outputs and workspaces allocated where the
caller passes none, and every computation runs in the HIP kernels of libmaestro.so on the current stream. There is no
fallback. Nothing here is recorded for autograd.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import _train
from ._native import _check, _dev, _ptr, _scratch, _shape, _stream, _Tensor, _workspace
from ._train import _DTYPE, _MOST, LayerGrad, _empties, _outputs

# Every function declared in include/maestro_layers.h.
EXPORTS = ("maestro_layer_grouped", "maestro_layer_grouped_grad_workspace", "maestro_layer_grouped_grad",
           "maestro_quantize_rows", "maestro_layer_int8", "maestro_pack_activations", "maestro_unpack_activations",
           "maestro_layer_grad_packed_workspace", "maestro_layer_grad_packed")

MAX_LAYER_GROUPS = 256
BLOCK = 32         # values of a row that share an exponent


class Quantized(NamedTuple):
    """Rows as signed bytes (``codes`` int8 [n][d]) with a ``scale`` each (float32 [n]): a value is code * scale."""
    codes: torch.Tensor
    scale: torch.Tensor


class Packed(NamedTuple):
    """Activations kept in 8 bits: ``codes`` [n][d], int8, or uint8 for rectified ones, and ``exponents`` uint8
    [n][ceil(d / 32)]: a value is code * 2^(exponent - 127)."""
    codes: torch.Tensor
    exponents: torch.Tensor


_lib = _tensors = None


def load():
    """libmaestro.so with the argument types of these operators set, and the native module given its entry points."""
    global _lib, _tensors
    if _lib is not None:
        return _lib
    lib = _train.load()
    P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.maestro_layer_grouped.argtypes = [i64, i32, i32, i32, i32, P, P, P, P, i32, P, P]
    lib.maestro_layer_grouped_grad_workspace.argtypes = [i64, i32, i32, i32, i32]
    lib.maestro_layer_grouped_grad.argtypes = [i64, i32, i32, i32, i32, P, P, P, P, i32, P, P, P, P, sz, P]
    lib.maestro_quantize_rows.argtypes = [i64, i32, i32, P, P, P, P]
    lib.maestro_layer_int8.argtypes = [i64, i32, i32, P, P, P, P, P, i32, i32, P, P]
    lib.maestro_pack_activations.argtypes = [i64, i32, i32, P, i32, P, P, P]
    lib.maestro_unpack_activations.argtypes = [i64, i32, i32, P, P, i32, P, P]
    lib.maestro_layer_grad_packed_workspace.argtypes = [i64, i32, i32, i32]
    lib.maestro_layer_grad_packed.argtypes = [i64, i32, i32, i32, P, P, i32, P, P, i32, P, P, P, P, sz, P]
    for f in EXPORTS:
        getattr(lib, f).restype = sz if f.endswith("_workspace") else ctypes.c_int
    module = _train._tensors
    module.bind_layers(*(ctypes.cast(getattr(lib, f), P).value for f in EXPORTS))      # in the order of its LayerEntries
    _tensors = module
    _lib = lib
    return lib


# As in ``_train``, a call goes to the native module first where outputs, workspace and stream are the binding's to choose, and is
# checked and made here only where that takes no part in it (None).


# what torch.cuda.current_device() and current_stream().cuda_stream come to, where this torch gives it away: looked up once, since
# a small call's time is the host's
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _here() -> int:
    """The current device's number."""
    return _device()


def _current(**tensors: Optional[torch.Tensor]) -> None:
    """Raise unless all are on the current device, where the kernels are launched."""
    here = _here()
    for name, t in tensors.items():
        if t is not None and t.get_device() != here:
            raise ValueError(f"{name} must be on the current device ({here}), is on {t.device}")


def _named(out: LayerGrad) -> dict:
    return {"out.x": out.x, "out.weight": out.weight, "out.bias": out.bias}


def _code(dtype, name: str) -> int:
    code = _DTYPE.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {dtype}")
    return code


def _matrix(t: torch.Tensor, name: str, *dtypes: torch.dtype):
    """(n, d) of a contiguous [n][d] tensor of one of these types."""
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d).replace('torch.', '') for d in dtypes)}, got {t.dtype}")
    _dev(t, name, t.dtype)
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError(f"{name} must be [n][d] with d >= 1")
    if t.shape[1] > _MOST:
        raise ValueError(f"{name} has more columns than an int32 counts")
    return t.shape


def _new(stream, device, *specs):
    """Uninitialised tensors of (shape, type), or None where None is given, for a call on ``stream``."""
    return _outputs(lambda: tuple(None if s is None else torch.empty(s[0], dtype=s[1], device=device) for s in specs), device, stream)


def _grouped_shapes(x: torch.Tensor, weight: torch.Tensor, offsets: torch.Tensor):
    code = _code(weight.dtype, "weight") if isinstance(weight, _Tensor) else None
    if code is None:
        raise TypeError("weight must be a float32 or bfloat16 tensor")
    _dev(weight, "weight", weight.dtype)
    _dev(x, "x", weight.dtype)
    if weight.dim() != 3 or x.dim() != 2 or x.shape[1] != weight.shape[2]:
        raise ValueError("x must be [n][d_in] and weight [groups][d_out][d_in]")
    groups, o, i = weight.shape
    if max(groups, o, i) > _MOST:
        raise ValueError("weight has more groups, rows or columns than an int32 counts")
    _shape(_dev(offsets, "offsets", torch.int64), "offsets", (groups + 1,))
    return code, x.shape[0], groups, i, o


def layer_grouped(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, offsets: torch.Tensor, relu: bool = True,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """maestro_layer_grouped: rows offsets[g] .. offsets[g + 1] of ``x`` [n][d_in] through group g's layer, in ``weight``
    [groups][d_out][d_in] (float32 or bfloat16) and ``bias`` [groups][d_out] (float32); ``offsets`` int64 [groups + 1] on
    the device. Rows of no group are left as they are in ``out`` (without one they hold whatever the memory held)."""
    lib = load()
    if out is None and stream is None:
        here = _here()
        got = _tensors.layer_grouped(x, weight, bias, offsets, relu, _raw_stream(here), here)
        if got is not None:
            return got
    dt, n, groups, i, o = _grouped_shapes(x, weight, offsets)
    _shape(_dev(bias, "bias", torch.float32), "bias", (groups, o))
    if out is None:
        out, = _empties(stream, x, ((n, o), 2))
    else:
        _shape(_dev(out, "out", weight.dtype), "out", (n, o))
    _current(x=x, weight=weight, bias=bias, offsets=offsets, out=out)
    st = lib.maestro_layer_grouped(n, groups, i, o, dt, _ptr(x), _ptr(weight), _ptr(bias), _ptr(offsets), int(bool(relu)),
                                   _ptr(out), _stream(stream))
    _check("maestro_layer_grouped", st)
    return out


def _grad_outputs(out: Optional[LayerGrad], want_x: bool, stream, x: torch.Tensor, dtype: torch.dtype, n: int, i: int,
                  weight_shape, bias_shape) -> LayerGrad:
    if out is None:
        return LayerGrad._make(_new(stream, x.device, ((n, i), dtype) if want_x else None, (weight_shape, torch.float32),
                                    (bias_shape, torch.float32)))
    if (out.x is not None) != bool(want_x):
        raise ValueError("out.x goes with want_x")
    if want_x:
        _shape(_dev(out.x, "out.x", dtype), "out.x", (n, i))
    _shape(_dev(out.weight, "out.weight", torch.float32), "out.weight", weight_shape)
    _shape(_dev(out.bias, "out.bias", torch.float32), "out.bias", bias_shape)
    return out


def layer_grouped_grad(x: torch.Tensor, weight: torch.Tensor, g_z: torch.Tensor, offsets: torch.Tensor,
                       relu_input: bool = False, want_x: bool = True, out: Optional[LayerGrad] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> LayerGrad:
    """maestro_layer_grouped_grad: gradients of a grouped layer given ``g_z`` [n][d_out], as ``layer_grad`` for every group:
    weights [groups][d_out][d_in] and biases [groups][d_out] in float32 (zeros for empty groups), and with ``want_x`` the
    input's. Rows of no group take no part, and theirs of ``out.x`` are left as they are."""
    lib = load()
    if out is None and workspace is None and stream is None:
        here = _here()
        got = _tensors.layer_grouped_grad(x, weight, g_z, offsets, relu_input, want_x, _raw_stream(here), here)
        if got is not None:
            return LayerGrad._make(got)
    dt, n, groups, i, o = _grouped_shapes(x, weight, offsets)
    _shape(_dev(g_z, "g_z", weight.dtype), "g_z", (n, o))
    out = _grad_outputs(out, want_x, stream, x, weight.dtype, n, i, (groups, o, i), (groups, o))
    _current(x=x, weight=weight, g_z=g_z, offsets=offsets, workspace=workspace, **_named(out))
    need = lib.maestro_layer_grouped_grad_workspace(n, groups, i, o, dt)
    _workspace(workspace)
    if workspace is None and need:
        workspace = _scratch(need, x.device, stream)
    st = lib.maestro_layer_grouped_grad(n, groups, i, o, dt, _ptr(x), _ptr(weight), _ptr(g_z), _ptr(offsets),
                                        int(bool(relu_input)), _ptr(out.x), _ptr(out.weight), _ptr(out.bias), _ptr(workspace),
                                        workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("maestro_layer_grouped_grad", st)
    return out


def quantize_rows(x: torch.Tensor, out: Optional[Quantized] = None, stream=None) -> Quantized:
    """maestro_quantize_rows: rows of ``x`` [n][d] (float32 or bfloat16) as signed bytes with a scale each, the largest
    magnitude over 127. Weights [d_out][d_in] so quantised have a scale for each output channel."""
    lib = load()
    if out is None and stream is None:
        here = _here()
        got = _tensors.quantize_rows(x, _raw_stream(here), here)
        if got is not None:
            return Quantized._make(got)
    n, d = _matrix(x, "x", torch.float32, torch.bfloat16)
    if out is None:
        out = Quantized._make(_new(stream, x.device, ((n, d), torch.int8), ((n,), torch.float32)))
    else:
        _shape(_dev(out.codes, "out.codes", torch.int8), "out.codes", (n, d))
        _shape(_dev(out.scale, "out.scale", torch.float32), "out.scale", (n,))
    _current(x=x, codes=out.codes, scale=out.scale)
    st = lib.maestro_quantize_rows(n, d, _DTYPE[x.dtype], _ptr(x), _ptr(out.codes), _ptr(out.scale), _stream(stream))
    _check("maestro_quantize_rows", st)
    return out


def layer_int8(x: Quantized, weight: Quantized, bias: torch.Tensor, relu: bool = True, dtype: torch.dtype = torch.bfloat16,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """maestro_layer_int8: y [n][d_out] = x weight^T + bias of quantised rows ``x`` and ``weight`` [d_out][d_in], rectified
    with ``relu``, in ``dtype`` (float32 or bfloat16; bias float32). Products are summed in whole numbers."""
    lib = load()
    dt = _code(dtype, "dtype")
    if out is None and stream is None:
        here = _here()
        got = _tensors.layer_int8(x.codes, x.scale, weight.codes, weight.scale, bias, relu, dt, _raw_stream(here), here)
        if got is not None:
            return got
    n, i = _matrix(x.codes, "x.codes", torch.int8)
    o, columns = _matrix(weight.codes, "weight.codes", torch.int8)
    if columns != i:
        raise ValueError("x must be [n][d_in] and weight [d_out][d_in]")
    if o > _MOST:
        raise ValueError("weight.codes has more rows than an int32 counts")
    _shape(_dev(x.scale, "x.scale", torch.float32), "x.scale", (n,))
    _shape(_dev(weight.scale, "weight.scale", torch.float32), "weight.scale", (o,))
    _shape(_dev(bias, "bias", torch.float32), "bias", (o,))
    if out is None:
        out, = _new(stream, x.codes.device, ((n, o), dtype))
    else:
        _shape(_dev(out, "out", dtype), "out", (n, o))
    _current(x=x.codes, x_scale=x.scale, weight=weight.codes, weight_scale=weight.scale, bias=bias, out=out)
    st = lib.maestro_layer_int8(n, i, o, _ptr(x.codes), _ptr(x.scale), _ptr(weight.codes), _ptr(weight.scale), _ptr(bias),
                                int(bool(relu)), dt, _ptr(out), _stream(stream))
    _check("maestro_layer_int8", st)
    return out


def _packed_shapes(packed: Packed):
    """(n, d, rectified) of a checkpoint."""
    n, d = _matrix(packed.codes, "codes", torch.int8, torch.uint8)
    _shape(_dev(packed.exponents, "exponents", torch.uint8), "exponents", (n, -(-d // BLOCK)))
    return n, d, int(packed.codes.dtype == torch.uint8)


def pack_activations(x: torch.Tensor, rectified: bool = False, out: Optional[Packed] = None, stream=None) -> Packed:
    """maestro_pack_activations: ``x`` [n][d] (float32 or bfloat16) in 8 bits, 32 values of a row to a power of two;
    ``rectified``: unsigned codes, 0 where x is not positive and at least 1 where it is."""
    lib = load()
    if out is None and stream is None:
        here = _here()
        got = _tensors.pack(x, rectified, _raw_stream(here), here)
        if got is not None:
            return Packed._make(got)
    n, d = _matrix(x, "x", torch.float32, torch.bfloat16)
    if out is None:
        out = Packed._make(_new(stream, x.device, ((n, d), torch.uint8 if rectified else torch.int8),
                                ((n, -(-d // BLOCK)), torch.uint8)))
    elif _packed_shapes(out) != (n, d, int(bool(rectified))):
        raise ValueError("out must have x's shape, and uint8 codes with rectified, int8 ones without")
    _current(x=x, codes=out.codes, exponents=out.exponents)
    st = lib.maestro_pack_activations(n, d, _DTYPE[x.dtype], _ptr(x), int(bool(rectified)), _ptr(out.codes), _ptr(out.exponents),
                                      _stream(stream))
    _check("maestro_pack_activations", st)
    return out


def unpack_activations(packed: Packed, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """maestro_unpack_activations: the values of a checkpoint in ``dtype`` (float32 or bfloat16), exactly."""
    lib = load()
    dt = _code(dtype, "dtype")
    if out is None and stream is None:
        here = _here()
        got = _tensors.unpack(packed.codes, packed.exponents, dt, _raw_stream(here), here)
        if got is not None:
            return got
    n, d, rectified = _packed_shapes(packed)
    if out is None:
        out, = _new(stream, packed.codes.device, ((n, d), dtype))
    else:
        _shape(_dev(out, "out", dtype), "out", (n, d))
    _current(codes=packed.codes, exponents=packed.exponents, out=out)
    st = lib.maestro_unpack_activations(n, d, dt, _ptr(packed.codes), _ptr(packed.exponents), rectified, _ptr(out), _stream(stream))
    _check("maestro_unpack_activations", st)
    return out


def layer_grad_packed(packed: Packed, weight: torch.Tensor, g_z: torch.Tensor, relu_input: bool = False, want_x: bool = True,
                      out: Optional[LayerGrad] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> LayerGrad:
    """maestro_layer_grad_packed: ``layer_grad`` of an input kept as ``packed``: the gradients for the values that
    ``unpack_activations`` gives. ``relu_input`` needs rectified (uint8) codes."""
    lib = load()
    if out is None and workspace is None and stream is None:
        here = _here()
        got = _tensors.layer_grad_packed(packed.codes, packed.exponents, weight, g_z, relu_input, want_x, _raw_stream(here), here)
        if got is not None:
            return LayerGrad._make(got)
    n, i, rectified = _packed_shapes(packed)
    if not isinstance(weight, _Tensor):
        raise TypeError("weight must be a float32 or bfloat16 tensor")
    dt = _code(weight.dtype, "weight")
    _dev(weight, "weight", weight.dtype)
    if weight.dim() != 2 or weight.shape[1] != i:
        raise ValueError("codes must be [n][d_in] and weight [d_out][d_in]")
    o = weight.shape[0]
    if o > _MOST:
        raise ValueError("weight has more rows than an int32 counts")
    if relu_input and not rectified:
        raise ValueError("relu_input needs rectified codes (uint8)")
    _shape(_dev(g_z, "g_z", weight.dtype), "g_z", (n, o))
    out = _grad_outputs(out, want_x, stream, g_z, weight.dtype, n, i, (o, i), (o,))
    _current(codes=packed.codes, exponents=packed.exponents, weight=weight, g_z=g_z, workspace=workspace, **_named(out))
    need = lib.maestro_layer_grad_packed_workspace(n, i, o, dt)
    _workspace(workspace)
    if workspace is None and need:
        workspace = _scratch(need, g_z.device, stream)
    st = lib.maestro_layer_grad_packed(n, i, o, dt, _ptr(packed.codes), _ptr(packed.exponents), rectified, _ptr(weight),
                                       _ptr(g_z), int(bool(relu_input)), _ptr(out.x), _ptr(out.weight), _ptr(out.bias),
                                       _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("maestro_layer_grad_packed", st)
    return out
