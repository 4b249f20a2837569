"""A call whose entry point reports a failed launch raises, and is made once: part of its work may be on the stream
already, and clipping in place a second time would scale what is already scaled."""
import ctypes

import pytest
import torch

import paper_2606_12950_amd as M
from paper_2606_12950_amd import _train

pytestmark = pytest.mark.gpu
ENTRIES = ("maestro_layer", "maestro_layer_grad_workspace", "maestro_layer_grad", "maestro_logprobs_workspace", "maestro_logprobs",
           "maestro_logprobs_grad", "maestro_clip_gradients_workspace", "maestro_clip_gradients")
LAUNCH = 4


def _calls():
    n, i, o = 8, 32, 16
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    x, w, b, g, t, s, h = z(n, i), z(o, i), z(o), z(n, o), z(n, dtype=torch.int32), z(n, 2), z(n)
    return {
        "maestro_logprobs": lambda: M.logprobs(g, t, k=3),
        "maestro_logprobs_grad": lambda: M.logprobs_grad(g, t, s, h, h, h),
        "maestro_layer": lambda: M.layer(x, w, b),
        "maestro_layer_grad": lambda: M.layer_grad(x, w, g),
        "maestro_clip_gradients": lambda: M.clip_gradients([x, w], 1.0),
    }


CALLS = ("maestro_logprobs", "maestro_logprobs_grad", "maestro_layer", "maestro_layer_grad", "maestro_clip_gradients")


@pytest.mark.parametrize("status", [1, 2, 3, LAUNCH])
@pytest.mark.parametrize("name", CALLS)
def test_a_failed_launch_is_not_made_again(name, status, monkeypatch):
    """The entry point is replaced by one that launches nothing and returns a status; the binding's own path counts too."""
    lib, made = _train.load(), []
    call = _calls()[name]

    def report(*args):
        made.append(name)
        return status

    stub = ctypes.CFUNCTYPE(ctypes.c_int, *getattr(lib, name).argtypes)(report)
    at = lambda f: ctypes.cast(stub if f == name else getattr(lib, f), ctypes.c_void_p).value
    real = [ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in ENTRIES]
    addresses = [at(f) for f in ENTRIES]
    monkeypatch.setattr(lib, name, report)
    try:
        _bind(addresses)
        with pytest.raises(M.MaestroError) as e:
            call()
    finally:
        _bind(real)
    assert len(made) == (1 if status == LAUNCH else 2)
    assert e.value.status == status and name in str(e.value)


def _bind(addresses):
    _train._tensors.bind(*addresses, M.MaestroError)
