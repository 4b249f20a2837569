"""maestro_clip_gradients against float64 on the CPU. Squares and their sum are float64, so the norm is the
float64 one rounded to float32 (2^-24 of itself) whatever the order; a scaled value is one float64
product rounded to float32 and then to its type: 2^-23 and, for bfloat16, 2^-8 of itself."""
import math

import pytest
import torch

import paper_2606_12950_amd as M

pytestmark = pytest.mark.gpu
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def make(sizes, seed, scale=1e-3, mixed=True):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g) * scale).to(torch.bfloat16 if mixed and i % 2 else torch.float32)
            for i, s in enumerate(sizes)]


def norm_of(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def check(ts, max_norm, in_place, views=None):
    dev = views if views is not None else [t.cuda() for t in ts]
    out = None if in_place else [torch.full_like(t, 5.0) for t in dev]
    got = M.clip_gradients(dev, max_norm, out=out)
    torch.cuda.synchronize()
    norm = norm_of(ts)
    assert abs(got.item() - norm) <= 2.0 ** -23 * norm
    scale = max_norm / norm if norm > max_norm else 1.0
    for a, t in zip(dev if in_place else out, ts):
        want = t.double() * scale
        if scale == 1.0:
            assert torch.equal(a.cpu(), t)
        else:
            assert ((a.cpu().double() - want).abs() <= ROUND[t.dtype] * want.abs() + 1e-44).all()
    if not in_place:
        for a, t in zip(dev, ts):
            assert torch.equal(a.cpu(), t)


SIZES = [[1], [2, 1], [0, 5, 0], [7, 8, 9, 15, 16, 17], [255, 256, 257, 1023], [16383, 16384, 16385], [100003], [1 << 20, 3, 1 << 18],
         [262144, 1024, 1048576, 1024, 65536, 64], list(range(1, 301)), [64] * 97, [5] * 1000, [3, 4_000_001, 1, 2_000_003]]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_sizes(sizes, in_place):
    print(f"clip {len(sizes)} tensors in_place={in_place}", flush=True)
    ts = make(sizes, len(sizes))
    n = norm_of(ts)
    for max_norm in (0.3 * n, 2.0 * n, 0.0):
        check(ts, max_norm, in_place)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_views_of_one_buffer_at_odd_places(dtype):
    sizes = [1, 3, 16384, 7, 1, 40001, 5, 2, 16383, 9]
    flat = (torch.randn(sum(sizes) + 4, generator=torch.Generator().manual_seed(1))).to(dtype)
    for in_place in (True, False):
        d = flat.cuda()
        views = list(d[1:-3].split(sizes))
        print(f"clip views {dtype} in_place={in_place}", flush=True)
        check(list(flat[1:-3].split(sizes)), 3.0, in_place, views)
        assert torch.equal(d[:1].cpu(), flat[:1]) and torch.equal(d[-3:].cpu(), flat[-3:])


def test_output_at_another_alignment():
    t = make([50001], 4, mixed=False)
    buf = torch.full((50005,), 5.0, device="cuda")
    M.clip_gradients([t[0].cuda()], 0.01, out=[buf[3:50004]])
    want = t[0].double() * (0.01 / norm_of(t))
    assert ((buf[3:50004].cpu().double() - want).abs() <= 2.0 ** -23 * want.abs()).all()
    assert (buf[:3] == 5.0).all() and buf[50004] == 5.0


def test_extreme_values():
    for scale in (1e30, 1e-30, 1e-39):      # squares out of float32's range on either side
        t = [torch.tensor([3.0, -4.0, 0.0] * 700) * scale]
        check(t, norm_of(t) * 1e-3, True)
    big = [torch.full((10,), 3e38), torch.full((3,), 3e38)]      # the norm itself is past float32
    d = [b.cuda() for b in big]
    assert M.clip_gradients(d, 1.0).item() == math.inf
    for a, b in zip(d, big):
        want = b.double() / norm_of(big)
        assert ((a.cpu().double() - want).abs() <= 2.0 ** -23 * want).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_norms_that_are_not_finite_scale_nothing(bad):
    for at in (0, 1):
        ts = make([1000, 70001], 3)
        ts[at][-1] = bad
        d = [t.cuda() for t in ts]
        out = [torch.empty_like(t) for t in d]
        for kw in (dict(), dict(out=out)):
            n = M.clip_gradients(d, 1e-3, **kw).item()
            assert math.isnan(n) if math.isnan(bad) else n == math.inf
            for t, a in zip(ts, kw.get("out", d)):
                assert torch.equal(a.cpu().view(torch.int16 if a.element_size() == 2 else torch.int32),
                                   t.view(torch.int16 if t.element_size() == 2 else torch.int32))


def test_norm_alone():
    ts = make([1000, 0, 33, 70001], 3)
    d = [t.cuda() for t in ts]
    n = M.gradient_norm(d)
    assert abs(n.item() - norm_of(ts)) <= 2.0 ** -23 * norm_of(ts)
    for a, t in zip(d, ts):
        assert torch.equal(a.cpu(), t)
    assert M.gradient_norm([torch.zeros(0, device="cuda")]).item() == 0.0
    assert M.clip_gradients([torch.zeros(5, device="cuda")], 0.0).item() == 0.0


def test_more_values_than_32_bits_count():
    n = (1 << 31) + 4099
    t = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    t[-1] = 1.0
    norm = math.sqrt((n - 1) * 2.0 ** -20 + 1.0)
    got = M.clip_gradients([t], norm / 4)
    assert abs(got.item() - norm) <= 2.0 ** -23 * norm
    assert (t[:-1] == 2.0 ** -12).all() and t[-1] == 0.25


def test_graph_equal_bits_and_side_stream():
    ts = [t.cuda() for t in make([1000, 5, 300001] + [77] * 200, 5)]
    out = [torch.empty_like(t) for t in ts]
    norm = torch.empty(1, device="cuda")
    ws = torch.empty(M._train.load().maestro_clip_gradients_workspace(len(ts)), dtype=torch.uint8, device="cuda")
    want_norm = M.clip_gradients(ts, 0.1, out=out).clone()
    want = [t.clone() for t in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = M.clip_gradients(ts, 0.1, out=out, stream=side)
    side.synchronize()
    assert torch.equal(again, want_norm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.clip_gradients(ts, 0.1, out=out, norm=norm, workspace=ws)
    for rep in range(3):
        for t in (*out, norm, ws):
            t.fill_(1)
        if rep == 1:
            M.gradient_norm(ts)
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want_norm)
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_refusals():
    f = torch.zeros(6, device="cuda")
    for bad, err in ((lambda: M.clip_gradients([], 1.0), ValueError), (lambda: M.clip_gradients([f.half()], 1.0), TypeError),
                     (lambda: M.clip_gradients([f.cpu()], 1.0), TypeError), (lambda: M.clip_gradients([f[::2]], 1.0), ValueError),
                     (lambda: M.clip_gradients([f], -1.0), ValueError), (lambda: M.clip_gradients([f], math.nan), ValueError),
                     (lambda: M.clip_gradients([f], 1.0, out=[f, f]), ValueError),
                     (lambda: M.clip_gradients([f], 1.0, out=[f.bfloat16()]), ValueError)):
        with pytest.raises(err):
            bad()


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("count", [12, 13, 159, 160, 161, 321])
def test_tables_just_full(count, in_place):
    """Counts around the tables' sizes; lengths around a unit of work (8,192 float32, 16,384 bfloat16)."""
    lengths = [1, 8191, 8192, 8193, 16383, 16384, 16385, 0, 32769, 77]
    ts = make([lengths[i % 10] for i in range(count)], count)
    print(f"clip tables of {count}", flush=True)
    total = math.sqrt(sum(float(t.double().square().sum()) for t in ts))
    dev = [t.cuda() for t in ts]
    out = None if in_place else [torch.empty_like(t) for t in dev]
    norm = M.clip_gradients(dev, total / 3, out=out)
    assert abs(float(norm) - total) <= 2.0 ** -22 * total
    for t, o in zip(ts, dev if in_place else out):
        want = t.double() / 3
        assert ((o.cpu().double() - want).abs() <= (2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -22) * want.abs() + 1e-38).all()
