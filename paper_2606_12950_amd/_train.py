"""Thin ctypes binding of the training operators (include/maestro_train.h).

Argument marshalling only, in the manner of ``_native``: the tensors are checked, outputs and
workspaces allocated where the caller passes none, and every computation runs in the HIP kernels of
libmaestro.so on the current stream. Where Python would take longer than the GPU (hundreds of tensors,
several outputs) the native module ``_tensors`` does it. There is no fallback.

Nothing here is recorded for autograd: a tensor that requires gradients is read as any other, and the results
are detached. ``logprobs_grad`` and ``layer_grad`` are the gradients.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import NamedTuple, Optional, Sequence

import torch

from . import _native
from ._native import MAESTRO_BF16, MAESTRO_F32, MaestroError, _check, _dev, _outputs, _ptr, _scratch, _shape, _stream, _Tensor, _workspace

# Every function declared in include/maestro_train.h.
EXPORTS = ("maestro_logprobs_workspace", "maestro_logprobs", "maestro_logprobs_grad", "maestro_layer",
           "maestro_layer_grad_workspace", "maestro_layer_grad", "maestro_clip_gradients_workspace",
           "maestro_clip_gradients")

MAX_ALTERNATIVES = 16

TENSORS_PATH = os.path.join(os.path.dirname(_native.LIBRARY_PATH), "_tensors.so")

_MOST = (1 << 31) - 1      # of an int32 argument: ctypes would cut a larger number off

_DTYPE = {torch.float32: MAESTRO_F32, torch.bfloat16: MAESTRO_BF16}


class Logprobs(NamedTuple):
    """Outputs of ``logprobs``; ``stats`` [n][2] are the row maxima and the logs of the sums of
    exponentials less the maximum, for ``logprobs_grad``. What was not asked for is None."""
    logprob: Optional[torch.Tensor]
    entropy: Optional[torch.Tensor]
    top_id: torch.Tensor
    top_logprob: torch.Tensor
    stats: Optional[torch.Tensor]


class LayerGrad(NamedTuple):
    """Outputs of ``layer_grad``: ``x`` in the layer's type (None where not wanted), ``weight`` and
    ``bias`` float32."""
    x: Optional[torch.Tensor]
    weight: torch.Tensor
    bias: torch.Tensor


_lib = _tensors = None


def load():
    """libmaestro.so with the argument types of the training operators set, and the binding's host half."""
    global _lib, _tensors
    if _lib is not None:
        return _lib
    lib = _native.load()
    if not os.path.exists(TENSORS_PATH):
        raise RuntimeError(f"{TENSORS_PATH} is missing: build it first (python -m paper_2606_12950_amd.build)")
    try:
        from . import _tensors as module
        built = module.torch_version
    except (ImportError, AttributeError) as e:         # a symbol that this torch does not have, or an older build
        built = str(e)
    if built != torch.__version__:
        raise RuntimeError(f"{TENSORS_PATH} was built against another torch ({built}) than {torch.__version__}: "
                           "build it again (python -m paper_2606_12950_amd.build)")
    P, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    lib.maestro_logprobs_workspace.argtypes = [i64, i32, i32, i32]
    lib.maestro_logprobs.argtypes = [i64, i32, P, i64, i32, P, i32, P, P, P, P, P, P, sz, P]
    lib.maestro_logprobs_grad.argtypes = [i64, i32, P, i64, i32, P, P, P, P, P, P, i64, P]
    lib.maestro_layer.argtypes = [i64, i32, i32, i32, P, P, P, i32, P, P]
    lib.maestro_layer_grad_workspace.argtypes = [i64, i32, i32, i32]
    lib.maestro_layer_grad.argtypes = [i64, i32, i32, i32, P, P, P, i32, P, P, P, P, sz, P]
    lib.maestro_clip_gradients_workspace.argtypes = [i32]
    lib.maestro_clip_gradients.argtypes = [i32, P, P, P, P, f32, P, P, sz, P]
    for f in EXPORTS:
        getattr(lib, f).restype = sz if f.endswith("_workspace") else ctypes.c_int
    module.bind(*(ctypes.cast(getattr(lib, f), P).value for f in (
        "maestro_layer", "maestro_layer_grad_workspace", "maestro_layer_grad", "maestro_logprobs_workspace", "maestro_logprobs",
        "maestro_logprobs_grad", "maestro_clip_gradients_workspace", "maestro_clip_gradients")), MaestroError)
    _tensors = module
    _lib = lib
    return lib


# The calls below go to the native module first where the outputs, the workspace and the stream are the binding's to choose: it
# takes a plain call whole and gives None for any other, and for one that the entry point's checks refuse; their errors are raised
# here. Host time, launch included (us, and without it): log probabilities of one token 8.3 (10.7), their gradient 4.5 (8.1), a
# layer 4.9 (7.0), its gradients 6.0 (9.0).


def _rows(t: torch.Tensor, name: str):
    """(dtype code, n, v, row stride) of a [n][v] float32 or bfloat16 tensor whose rows are contiguous and do
    not overlap."""
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    shape = t.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError(f"{name} must be [n][v] with v >= 1")
    n, v = shape
    if v > _MOST:
        raise ValueError(f"{name} has more columns than an int32 counts")
    stride, inner = t.stride()
    if n <= 1:
        stride = v
    if (v > 1 and inner != 1) or stride < v:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return code, n, v, stride


def _empties(stream, like: torch.Tensor, *specs):
    """The native module's ``empties`` for a call on ``stream``."""
    return _outputs(lambda: _tensors.empties(like, *specs), like.device, stream)


def logprobs(logits: torch.Tensor, token: Optional[torch.Tensor] = None, k: int = 0, want_entropy: bool = True,
             want_stats: bool = True, out: Optional[Logprobs] = None, workspace: Optional[torch.Tensor] = None,
             stream=None) -> Logprobs:
    """maestro_logprobs: for every row of ``logits`` [n][v] (float32 or bfloat16; rows may lie in a wider
    array) the log probability of its ``token`` (int32 [n], outside [0, v): none, 0), the entropy, the
    ``k`` likeliest tokens with their log probabilities, and the row statistics. -inf masks a logit."""
    lib = load()
    if out is None and workspace is None and stream is None:
        got = _tensors.logprobs(logits, token, k, want_entropy, want_stats, _stream(None))
        if got is not None:
            return Logprobs._make(got)
    dt, n, v, stride = _rows(logits, "logits")
    dev = logits.device
    if not 0 <= k <= MAX_ALTERNATIVES:
        raise ValueError(f"k must be 0 .. {MAX_ALTERNATIVES}")
    if token is not None:
        _shape(_dev(token, "token", torch.int32), "token", (n,))
    if out is None:
        row = ((n,), 0)
        out = Logprobs._make(_empties(stream, logits, row if token is not None else None, row if want_entropy else None,
                                      ((n, k), 1), ((n, k), 0), ((n, 2), 0) if want_stats else None))
    else:
        if (out.logprob is None) != (token is None):
            raise ValueError("logprob goes with token")
        for t, name, shape in ((out.logprob, "logprob", (n,)), (out.entropy, "entropy", (n,)), (out.stats, "stats", (n, 2))):
            if t is not None:
                _shape(_dev(t, name, torch.float32), name, shape)
        if k or out.top_id is not None:
            _shape(_dev(out.top_id, "top_id", torch.int32), "top_id", (n, k))
        if k or out.top_logprob is not None:
            _shape(_dev(out.top_logprob, "top_logprob", torch.float32), "top_logprob", (n, k))
    need = lib.maestro_logprobs_workspace(n, v, k, dt)
    _workspace(workspace)
    if workspace is None and need:
        workspace = _scratch(need, dev, stream)
    st = lib.maestro_logprobs(n, v, _ptr(logits), stride, dt, _ptr(token), k, _ptr(out.logprob),
                              _ptr(out.entropy), _ptr(out.top_id), _ptr(out.top_logprob), _ptr(out.stats),
                              _ptr(workspace), workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("maestro_logprobs", st)
    return out


def logprobs_grad(logits: torch.Tensor, token: Optional[torch.Tensor], stats: torch.Tensor,
                  entropy: Optional[torch.Tensor], g_logprob: Optional[torch.Tensor],
                  g_entropy: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """maestro_logprobs_grad: the gradient with respect to the logits of the sums of ``g_logprob`` times
    the log probabilities and ``g_entropy`` times the entropies (float32 [n], either may be None), in the
    logits' type. ``stats`` and ``entropy`` are what ``logprobs`` returned; ``out`` may be ``logits``."""
    lib = load()
    if out is None and stream is None:
        got = _tensors.logprobs_grad(logits, token, stats, entropy, g_logprob, g_entropy, _stream(None))
        if got is not None:
            return got
    dt, n, v, stride = _rows(logits, "logits")
    if (token is None) != (g_logprob is None) or (g_logprob is None and g_entropy is None):
        raise ValueError("g_logprob goes with token, and one of g_logprob and g_entropy is needed")
    if g_entropy is not None and entropy is None:
        raise ValueError("g_entropy needs the entropies")
    if token is not None:
        _shape(_dev(token, "token", torch.int32), "token", (n,))
    _shape(_dev(stats, "stats", torch.float32), "stats", (n, 2))
    for t, name in ((entropy, "entropy"), (g_logprob, "g_logprob"), (g_entropy, "g_entropy")):
        if t is not None:
            _shape(_dev(t, name, torch.float32), name, (n,))
    if out is None:
        (out,), out_stride = _empties(stream, logits, ((n, v), 2)), v
    else:
        *same, out_stride = _rows(out, "out")
        if same != [dt, n, v]:
            raise ValueError("out must have the logits' shape and type")
    st = lib.maestro_logprobs_grad(n, v, _ptr(logits), stride, dt, _ptr(token), _ptr(stats), _ptr(entropy),
                                   _ptr(g_logprob), _ptr(g_entropy), _ptr(out), out_stride, _stream(stream))
    _check("maestro_logprobs_grad", st)
    return out


def _layer_shapes(x: torch.Tensor, weight: torch.Tensor):
    code = _DTYPE.get(weight.dtype) if isinstance(weight, torch.Tensor) else None
    if code is None:
        raise TypeError("weight must be a float32 or bfloat16 tensor")
    _dev(weight, "weight", weight.dtype)
    _dev(x, "x", weight.dtype)
    if weight.dim() != 2 or x.dim() != 2 or x.shape[1] != weight.shape[1]:
        raise ValueError("x must be [n][d_in] and weight [d_out][d_in]")
    o, i = weight.shape
    if o > _MOST or i > _MOST:
        raise ValueError("weight has more rows or columns than an int32 counts")
    return code, x.shape[0], i, o


def layer(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, relu: bool = True,
          out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """maestro_layer: y [n][d_out] = x weight^T + bias, rectified with ``relu``, in the weights' type
    (float32 or bfloat16; bias float32). Widths are multiples of 16."""
    lib = load()
    if out is None and stream is None:
        got = _tensors.layer(x, weight, bias, relu, _stream(None))
        if got is not None:
            return got
    dt, n, i, o = _layer_shapes(x, weight)
    _shape(_dev(bias, "bias", torch.float32), "bias", (o,))
    if out is None:
        out, = _empties(stream, x, ((n, o), 2))
    else:
        _shape(_dev(out, "out", weight.dtype), "out", (n, o))
    st = lib.maestro_layer(n, i, o, dt, _ptr(x), _ptr(weight), _ptr(bias), int(bool(relu)), _ptr(out), _stream(stream))
    _check("maestro_layer", st)
    return out


def layer_grad(x: torch.Tensor, weight: torch.Tensor, g_z: torch.Tensor, relu_input: bool = False,
               want_x: bool = True, out: Optional[LayerGrad] = None, workspace: Optional[torch.Tensor] = None,
               stream=None) -> LayerGrad:
    """maestro_layer_grad: gradients of z = x weight^T + bias given ``g_z`` [n][d_out]: those of the weights and
    biases in float32, and with ``want_x`` the input's in the layer's type, 0 where x <= 0 with
    ``relu_input`` (x the output of a rectified layer: the result is the gradient of that layer's z)."""
    lib = load()
    if out is None and workspace is None and stream is None:
        got = _tensors.layer_grad(x, weight, g_z, relu_input, want_x, _stream(None))
        if got is not None:
            return LayerGrad._make(got)
    dt, n, i, o = _layer_shapes(x, weight)
    _shape(_dev(g_z, "g_z", weight.dtype), "g_z", (n, o))
    dev = x.device
    if out is None:
        out = LayerGrad._make(_empties(stream, x, ((n, i), 2) if want_x else None, ((o, i), 0), ((o,), 0)))
    else:
        if (out.x is not None) != want_x:
            raise ValueError("out.x goes with want_x")
        if want_x:
            _shape(_dev(out.x, "out.x", weight.dtype), "out.x", (n, i))
        _shape(_dev(out.weight, "out.weight", torch.float32), "out.weight", (o, i))
        _shape(_dev(out.bias, "out.bias", torch.float32), "out.bias", (o,))
    need = lib.maestro_layer_grad_workspace(n, i, o, dt)
    _workspace(workspace)
    if workspace is None and need:
        workspace = _scratch(need, dev, stream)
    st = lib.maestro_layer_grad(n, i, o, dt, _ptr(x), _ptr(weight), _ptr(g_z), int(bool(relu_input)), _ptr(out.x),
                                _ptr(out.weight), _ptr(out.bias), _ptr(workspace),
                                workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("maestro_layer_grad", st)
    return out


def clip_gradients(tensors: Sequence[torch.Tensor], max_norm: float, out: Optional[Sequence[torch.Tensor]] = None,
                   norm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """maestro_clip_gradients: scales all ``tensors`` (float32 or bfloat16, contiguous) by max_norm / norm where
    the norm of all their values together exceeds ``max_norm``, in place or into ``out``. Returns the
    norm before clipping, float32 [1] on the device. A norm that is not finite scales nothing. ``max_norm`` past
    float32's range (math.inf) computes the norm alone and takes no ``out``. No two tensors overlap."""
    lib = load()
    tensors = list(tensors)
    if not tensors:
        raise ValueError("at least one tensor")
    max_norm = float(max_norm)
    if not max_norm >= 0.0:
        raise ValueError("max_norm must not be negative or NaN")
    out = None if out is None else list(out)
    if norm is None and workspace is None and stream is None:
        got = _tensors.clip(tensors, max_norm, out, _stream(None))
        if got is not None:
            return got
    at, sizes, codes = _tensors.table(tensors, "tensors")
    count, oat = len(tensors), None
    if out is not None:
        oat, osizes, ocodes = _tensors.table(out, "out")
        if osizes != sizes or ocodes != codes:
            raise ValueError("out must have one output per tensor, of its size and type")
    dev = tensors[0].device
    if norm is None:
        norm, = _empties(stream, tensors[0], ((1,), 0))
    else:
        _shape(_dev(norm, "norm", torch.float32), "norm", (1,))
    _workspace(workspace)
    if workspace is None:
        workspace = _scratch(lib.maestro_clip_gradients_workspace(count), dev, stream)
    st = lib.maestro_clip_gradients(count, at, oat, sizes, codes, max_norm, _ptr(norm), _ptr(workspace),
                                    workspace.numel(), _stream(stream))
    _check("maestro_clip_gradients", st)
    return norm


def gradient_norm(tensors: Sequence[torch.Tensor], norm: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The norm of ``clip_gradients`` alone; nothing is scaled."""
    return clip_gradients(tensors, math.inf, None, norm, workspace, stream)
