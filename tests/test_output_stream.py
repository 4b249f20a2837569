"""Outputs that the binding allocates for a call on a stream of the caller's: taken from that stream's pool, so that one
dropped early is not given to the current stream's next tensor while the call still writes it, and lent to the
current stream, so that the call's stream is not given it again before what the caller queued with it has run."""
import contextlib
import types

import pytest
import torch

import paper_2606_12950_amd as M
from paper_2606_12950_amd import _native, _train


def _calls(dev):
    """Every training call without outputs of the caller's."""
    n, i, o = 64, 32, 48
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device=dev)
    x, w, b, g, t, s, h = z(n, i), z(o, i), z(o), z(n, o), z(n, dtype=torch.int32), z(n, 2), z(n)
    return {
        "maestro_logprobs": lambda q: M.logprobs(g, t, k=3, stream=q),
        "maestro_logprobs without alternatives": lambda q: M.logprobs(g, want_stats=False, stream=q),
        "maestro_logprobs_grad": lambda q: (M.logprobs_grad(g, t, s, h, h, h, stream=q),),
        "maestro_layer": lambda q: (M.layer(x, w, b, stream=q),),
        "maestro_layer_grad": lambda q: M.layer_grad(x, w, g, stream=q),
        "maestro_clip_gradients": lambda q: (M.clip_gradients([x, w], 1.0, stream=q),),
    }


CALLS = sorted(_calls("cpu"))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("kind", ["torch", "handle"])
def test_outputs_are_taken_under_the_launch_stream(monkeypatch, name, kind):
    """On the CPU, the library, the streams and the allocator replaced by recorders."""
    class Stream:                             # stands for torch.cuda.Stream
        cuda_stream = 4096

    class External(Stream):
        def __init__(self, handle, device=None):
            self.cuda_stream = handle

    default = Stream()
    default.cuda_stream = 0
    current, taken, lent = [default], [], []

    @contextlib.contextmanager
    def on(s):
        old, current[0] = current[0], s
        yield
        current[0] = old

    class Made:
        is_cuda, shape = True, ()

        def record_stream(self, s):
            lent.append(s.cuda_stream)

        def data_ptr(self):
            return 4096

    def empties(like, *specs):
        taken.extend(current[0].cuda_stream for p in specs if p)
        return tuple(p and Made() for p in specs)

    call = _calls("cpu")[name]
    status = lambda *a: 0
    lib = types.SimpleNamespace(**{f: status for f in _train.EXPORTS})
    monkeypatch.setattr(_train, "load", lambda: lib)
    monkeypatch.setattr(_train, "_tensors", types.SimpleNamespace(empties=empties, table=lambda t, name: (b"", b"", b"")))
    monkeypatch.setattr(_train, "_dev", lambda t, *a: t)
    monkeypatch.setattr(_train, "_rows", lambda t, name: (0, *t.shape, t.shape[1]))
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", External)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[0])
    handle = Stream() if kind == "torch" else types.SimpleNamespace(cuda_stream=8192)
    made = [t for t in call(handle) if t is not None]
    assert taken == [handle.cuda_stream] * len(made)
    assert lent == [0] * len(made)


def _blocks(out):
    return {t.data_ptr() for t in out if t is not None and t.numel()}


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_neither_stream_is_given_the_blocks_too_soon(name):
    call = _calls("cuda")[name]
    side = torch.cuda.Stream()
    for q in (side, types.SimpleNamespace(cuda_stream=side.cuda_stream)):
        torch.cuda.synchronize()
        print(f"outputs {name} {type(q).__name__}", flush=True)
        out = call(q)
        sizes, at = [(t.numel(), t.dtype) for t in out if t is not None and t.numel()], _blocks(out)
        torch.cuda.synchronize()
        del out
        mine = [torch.empty(s, dtype=d, device="cuda") for s, d in sizes for _ in range(4)]
        assert not at & _blocks(mine)
        out = call(q)
        at = _blocks(out)
        torch.cuda._sleep(50_000_000)         # the caller's own work with them, on the current stream
        del out
        again = _blocks(call(q))
        assert not torch.cuda.current_stream().query()
        assert not at & again
    torch.cuda.synchronize()
