"""As test_output_stream, for the scheduler's calls: outputs that the binding allocates for a call on a stream of the caller's."""
import contextlib
import types

import pytest
import torch

import paper_2606_12950_amd as M
from paper_2606_12950_amd import _native
from test_output_stream import _blocks

i32, f32, f64, i64 = torch.int32, torch.float32, torch.float64, torch.int64


def _calls(dev):
    """Every call that allocates outputs, without outputs of the caller's; the inputs are made here, before a call."""
    n, m, k, w, win = 64, 16, 4, 32, 1000
    z = lambda *s, dtype=f32: torch.zeros(*s, dtype=dtype, device=dev)
    dims = (256, 512, 512, 64)
    ws = [z(o, i, dtype=torch.bfloat16) for i, o in zip(dims[:-1], dims[1:])]
    bs = [z(o) for o in dims[1:]]
    off = torch.arange(w + 1, dtype=i64, device=dev)
    ids, rows, kv, per_model = z(n, dtype=i32), z(n), z(n, dtype=f64), z(k)
    free, queue, mask = z(m, dtype=f64) + 1, z(m), z(m, dtype=i64)
    x, bins, role_head, heads, iso = z(n, 256, dtype=torch.bfloat16), z(64), z(1, dtype=i32) + 1, z(64), z(2)
    rtt, classes, bounds = z(1, m), z(1, 3), z(6)
    engines, no_level, no_bytes, no_cost = z(m + 1, dtype=i32), z(0, dtype=i32), z(0, dtype=f64), z(0)
    tier, size, bw, setup = z(m, k, dtype=torch.uint8), z(k, dtype=f64), z(5, dtype=f64) + 1, z(5)
    window, values, latency, deadline, lists = z(win, dtype=f64) + 1, z(win), z(w), z(w, dtype=i64), z(1 << 16, dtype=torch.uint8)
    return {
        "maestro_predict": lambda s: M.predict(x, ws, bs, bins, ids, ids, per_model, stream=s),
        "maestro_predict_two_phase": lambda s: M.predict_two_phase(x, ws, bs, role_head, heads, iso, iso, 100.0, ids, ids, ids, ids,
                                                                   per_model, stream=s),
        "maestro_route_ex": lambda s: M.route(ids, rows, kv, per_model, free, queue, queue, mask, k=2, stream=s),
        "maestro_route_fitness": lambda s: M.route_fitness(ids, ids, ids, kv, free, queue, queue, mask, queue, rtt, classes, bounds,
                                                           k, k=2, stream=s),
        "maestro_degradation_plans": lambda s: M.degradation_plans(engines, no_level, no_bytes, no_cost, 1.0, stream=s),
        "maestro_activation_latency": lambda s: (M.activation_latency(tier, size, bw, setup, stream=s),),
        "maestro_adaptive_rho": lambda s: M.adaptive_rho(window, window, 0.2, 0.9, stream=s),
        "maestro_quantiles": lambda s: (M.quantiles(values, stream=s),),
        "maestro_route_sort_nodes": lambda s: (M.route_sort_nodes(free, queue, queue, mask, k, stream=s),),
        "maestro_route_walk": lambda s: M.route_walk(ids, rows, kv, per_model, m, lists, k=2, stream=s),
        "maestro_prioritize": lambda s: M.prioritize(off, latency, deadline, 0, stream=s),
    }


CALLS = sorted(_calls("cpu"))


@pytest.mark.parametrize("name", CALLS)
def test_outputs_are_taken_under_the_launch_stream(monkeypatch, name):
    """On the CPU, the library, the streams and the allocator replaced by recorders."""
    class Stream:                             # stands for torch.cuda.Stream
        def __init__(self, handle=4096):
            self.cuda_stream = handle

    default = Stream(0)
    current, taken, lent = [default], [], []

    @contextlib.contextmanager
    def on(s):
        old, current[0] = current[0], s
        yield
        current[0] = old

    real_empty = torch.empty

    def empty(*a, **kw):
        taken.append(current[0].cuda_stream)
        return real_empty(*a, **kw)

    call = _calls("cpu")[name]

    class Library:                            # a status of 0 from every call, 64 KB for every workspace
        def __getattr__(self, f):
            return lambda *a: 65536 if "workspace" in f or f.endswith("_bytes") else 0

    monkeypatch.setattr(_native, "load", Library)
    monkeypatch.setattr(_native, "_dev", lambda t, *a: t)
    monkeypatch.setattr(_native, "_may_allocate", lambda stream: True)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[0])
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: lent.append(s.cuda_stream))
    made = [t for t in call(Stream()) if t is not None]
    assert set(taken) == {4096} and lent == [0] * len(made)


@pytest.mark.gpu
@pytest.mark.parametrize("name", [c for c in CALLS if c != "maestro_route_walk"])
def test_neither_stream_is_given_the_blocks_too_soon(name):
    call = _calls("cuda")[name]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    print(f"outputs {name}", flush=True)
    out = call(side)
    sizes, at = [(t.numel(), t.dtype) for t in out if t is not None and t.numel()], _blocks(out)
    torch.cuda.synchronize()
    del out
    mine = [torch.empty(s, dtype=d, device="cuda") for s, d in sizes for _ in range(4)]
    assert not at & _blocks(mine)
    out = call(side)
    at = _blocks(out)
    torch.cuda._sleep(50_000_000)             # the caller's own work with them, on the current stream
    del out
    again = _blocks(call(side))
    assert not torch.cuda.current_stream().query()
    assert not at & again
    torch.cuda.synchronize()
