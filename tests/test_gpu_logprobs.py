"""maestro_logprobs and maestro_logprobs_grad against the definition in float64 (torch on the CPU).

Bounds. x - m is exact to half an ulp, e^d by the hardware's 2^x to (|d| + 2) 2^-23 of itself, a sum of
v terms to at most 576 2^-24 of itself (chains of up to 512 additions, then a tree), its logarithm to 2 ulp: a log
probability l is off by at most 2^-24 (4 |l| + 640), an entropy h by 2^-24 (640 + 16 h) (1 + h). A
gradient's terms are products of p (off by 2^-23 (|ln p| + 8) of itself) and are rounded once to the type."""
import math

import pytest
import torch

import paper_2606_12950_amd as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}
INF = math.inf


def reference(x, token, k):
    """(logprob, entropy, ids, top, m, ln S) in float64."""
    x = x.double()
    n, v = x.shape
    m = x.amax(1)
    bad = torch.isnan(m) | (m == INF)
    none = m == -INF
    d = x - torch.where(none | bad, 0.0, m)[:, None]
    e = d.exp()
    ls = e.sum(1).log()
    lp = d - ls[:, None]
    p = lp.exp()
    h = -torch.where(p > 0, p * lp, 0.0).sum(1)
    t = token.long()
    given = (t >= 0) & (t < v)
    mine = torch.where(none, -INF, lp.gather(1, t.clamp(0, v - 1)[:, None])[:, 0])
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    top = lp.gather(1, order)
    hidden = x.gather(1, order) == -INF
    ids = torch.where(hidden, -1, order)
    top = torch.where(hidden, -INF, top)
    if k > v:
        ids = torch.cat([ids, torch.full((n, k - v), -1)], 1)
        top = torch.cat([top, torch.full((n, k - v), -INF, dtype=torch.float64)], 1)
    nan = math.nan
    mine = torch.where(given, torch.where(bad, nan, mine), 0.0)
    h = torch.where(bad, nan, torch.where(none, 0.0, h))
    ids = torch.where(bad[:, None], -1, ids)
    top = torch.where(bad[:, None], nan, top)
    return mine, h, ids.int(), top, torch.where(bad, nan, m), torch.where(bad, nan, ls)


def close(got, want, bound, what):
    got = got.cpu().double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = (got - want).abs()
    wrong = ~(same | (off <= bound))
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} off, first at {wrong.nonzero()[0].tolist()}: " \
        f"{got[wrong][0].item()} for {want[wrong][0].item()}"


def check(x, token, k, **kw):
    """x: a CPU tensor [n][v] (rows may be strided), checked on the GPU in the same layout."""
    dev = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda") if x.numel() else x.cuda()
    dev.copy_(x)
    got = M.logprobs(dev, token.cuda(), k=k, **kw)
    torch.cuda.synchronize()
    lp, h, ids, top, m, ls = reference(x, token, k)
    close(got.logprob, lp, U * (4 * lp.abs() + 640), "logprob")
    close(got.entropy, h, U * (640 + 16 * h) * (1 + h), "entropy")
    assert torch.equal(got.top_id.cpu(), ids), "ids"
    close(got.top_logprob, top, U * (4 * top.abs() + 640), "top_logprob")
    close(got.stats[:, 0], m, torch.zeros(()), "max")
    close(got.stats[:, 1], ls, U * (4 * ls.abs() + 640), "ln S")
    return got


def draw(n, v, dtype, seed, spread=2.5, masked=0.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.full((n, v + pad), math.nan, dtype=dtype)
    x = wide[:, :v]
    z = torch.randn(n, v, generator=g) * spread
    if masked:
        z[torch.rand(n, v, generator=g) < masked] = -INF
    x.copy_(z.to(dtype))
    return x, torch.randint(-1, v + 1, (n,), generator=g, dtype=torch.int32)


SIZES = [(1, 1), (5, 1), (3, 2), (1000, 2), (7, 3), (65, 7), (64, 8), (33, 16), (257, 31), (1023, 32), (4099, 64),
         (300, 65), (129, 100), (64, 127), (77, 128), (50, 200), (31, 255), (31, 256), (19, 257), (9, 511), (9, 512), (11, 513),
         (301, 1000), (5, 1024), (7, 1025), (6, 2047), (5, 4096), (300, 4099), (3, 8192), (2, 16385), (1, 32000),
         (3, 50257), (1, 65536), (1, 65537), (300, 32003), (1, 131072), (2, 131073), (1, 300001), (5, 262147)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v", SIZES)
def test_sizes(n, v, dtype):
    print(f"logprobs n={n} v={v} {dtype}", flush=True)
    x, token = draw(n, v, dtype, n * 31 + v)
    check(x, token, min(16, 4 + n % 5))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k", range(17))
@pytest.mark.parametrize("n,v", [(70, 5), (130, 64), (40, 300), (9, 3000), (3, 40001)])
def test_alternatives(n, v, k, dtype):
    print(f"logprobs n={n} v={v} k={k} {dtype}", flush=True)
    check(*draw(n, v, dtype, k + v, masked=0.3), k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [1, 6, 64, 72, 300, 2500, 40000, 140000])
def test_masks_ties_and_extremes(v, dtype):
    """Rows masked throughout or but for one place, of one value, of the type's lowest value, rising,
    falling, with huge ranges, signed zeros, NaN and +inf (here and there also beside masked places)."""
    print(f"logprobs extremes v={v} {dtype}", flush=True)
    low = torch.finfo(dtype).min
    rows = []
    z = torch.zeros(v)
    rows.append(torch.full((v,), -INF))
    for at in {0, v // 2, v - 1}:
        r = torch.full((v,), -INF)
        r[at] = 3.0
        rows.append(r)
    rows += [z.clone(), torch.full((v,), -7.25), torch.full((v,), low), torch.arange(v) / 16.0, -torch.arange(v) / 16.0]
    r = torch.full((v,), low)
    r[v // 3] = 0.5
    rows.append(r)
    r = torch.full((v,), -INF)
    r[v // 3] = low
    rows.append(r)
    r = z.clone()
    r[::2] = -0.0
    rows.append(r)
    r = z.clone()
    r[v - 1] = 1e30
    rows.append(r)
    rows.append(torch.full((v,), 3e38))
    for bad in (math.nan, INF):
        for at in {0, v // 2, v - 1}:
            r = torch.full((v,), -INF)
            r[at] = bad
            rows.append(r)
            r = torch.randn(v, generator=torch.Generator().manual_seed(at))
            r[at] = bad
            rows.append(r)
    r = z.clone()
    r[0], r[v - 1] = math.nan, INF
    rows.append(r)
    x = torch.stack(rows).to(dtype)
    n = x.shape[0]
    for token in (torch.zeros(n), torch.full((n,), v // 3), torch.full((n,), v - 1), torch.full((n,), -1),
                  torch.full((n,), v), torch.full((n,), 2 ** 31 - 1), torch.full((n,), -2 ** 31)):
        check(x, token.to(torch.int32), 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [64, 1000, 20000])
@pytest.mark.parametrize("pad", [1, 2, 5, 8, 13])
def test_strides(v, pad, dtype):
    print(f"logprobs stride v={v} pad={pad} {dtype}", flush=True)
    check(*draw(37, v, dtype, pad, masked=0.1, pad=pad), 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_unaligned_start(dtype):
    for v, shift in ((64, 1), (64, 3), (999, 1), (30001, 7)):
        base = torch.randn(9 * v + shift, generator=torch.Generator().manual_seed(v)).to(dtype)
        x = base[shift:].view(9, v)
        print(f"logprobs start v={v} shift={shift} {dtype}", flush=True)
        dev = base.cuda()[shift:].view(9, v)
        assert dev.data_ptr() % 16
        token = torch.arange(9, dtype=torch.int32)
        got = M.logprobs(dev, token.cuda(), k=3)
        lp, h, ids, top, _, _ = reference(x, token, 3)
        close(got.logprob, lp, U * (4 * lp.abs() + 640), "logprob")
        assert torch.equal(got.top_id.cpu(), ids)


def test_few_values_many_ties():
    g = torch.Generator().manual_seed(3)
    for dtype in (torch.float32, torch.bfloat16):
        for n, v in ((100, 64), (50, 700), (9, 9000), (2, 70000)):
            print(f"logprobs ties n={n} v={v} {dtype}", flush=True)
            x = torch.randint(-2, 3, (n, v), generator=g).to(dtype)
            check(x, torch.randint(0, v, (n,), generator=g, dtype=torch.int32), 16)


def test_large_logits_keep_their_precision():
    g = torch.Generator().manual_seed(5)
    for n, v in ((64, 64), (9, 3000)):
        x = torch.randn(n, v, generator=g) * 2 + 1000.0
        check(x, torch.randint(0, v, (n,), generator=g, dtype=torch.int32), 4)


def test_offsets_past_32_bits():
    stride = (1 << 30) + 8
    buf = torch.empty(2 * stride + 1000, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 1000), (stride, 1))
    z, token = draw(3, 1000, torch.bfloat16, 1)
    x.copy_(z)
    got = M.logprobs(x, token.cuda(), k=4)
    lp, _, ids, _, m, ls = reference(z, token, 4)
    close(got.logprob, lp, U * (4 * lp.abs() + 640), "logprob")
    assert torch.equal(got.top_id.cpu(), ids)
    g = torch.ones(3, device="cuda")
    M.logprobs_grad(x, token.cuda(), got.stats, None, g, out=x)
    close(x, grad_reference(z, token, g.cpu(), None)[0], grad_bound(z, token, g.cpu(), None), "grad")


def test_optional_outputs():
    x, token = draw(40, 64, torch.float32, 8)
    full = M.logprobs(x.cuda(), token.cuda(), k=2)
    a = M.logprobs(x.cuda(), k=2, want_entropy=False, want_stats=False)
    assert a.logprob is None and a.entropy is None and a.stats is None
    assert torch.equal(a.top_id, full.top_id) and torch.equal(a.top_logprob, full.top_logprob)
    b = M.logprobs(x.cuda(), token.cuda())
    assert b.top_id.shape == (40, 0) and torch.equal(b.logprob, full.logprob) and torch.equal(b.entropy, full.entropy)
    assert M.logprobs(x.cuda()[:0], token.cuda()[:0], k=3).top_id.shape == (0, 3)


# --- gradient ---------------------------------------------------------------------------------

def grad_reference(x, token, g, ge):
    x = x.double()
    v = x.shape[1]
    _, h, _, _, m, ls = reference(x, torch.full((x.shape[0],), -1), 0)
    lp = x - torch.where(torch.isinf(m), 0.0, m)[:, None] - ls[:, None]
    lp = torch.where((m == -INF)[:, None], -INF, lp)
    p = lp.exp()
    t = token.long()
    g = torch.where((t >= 0) & (t < v), g.double(), 0.0) if g is not None else torch.zeros(x.shape[0], dtype=torch.float64)
    ge = ge.double() if ge is not None else torch.zeros_like(g)
    hot = torch.zeros_like(x).scatter_(1, t.clamp(0, v - 1)[:, None], 1.0)
    plogp = torch.where(p > 0, p * lp.clamp_min(-1e300), 0.0)
    plogp = torch.where(torch.isnan(p), p, plogp)
    grad = g[:, None] * (hot - p) - torch.where(ge == 0, 0.0, ge)[:, None] * (plogp + p * torch.where(ge == 0, 0.0, h)[:, None])
    zero = (m == -INF) | ((g == 0) & (ge == 0))
    return torch.where(zero[:, None], 0.0, grad), p, lp, h, g, ge, hot


def grad_bound(x, token, g, ge):
    grad, p, lp, h, gg, gge, hot = grad_reference(x, token, g, ge)
    l = lp.abs().clamp_max(1e3)
    size = p * (gg.abs()[:, None] + gge.abs()[:, None] * (l + h.abs()[:, None] + 1))
    return size * 2.0 ** -22 * (l + 16) + hot * gg.abs()[:, None] * 2.0 ** -22 + HALF[x.dtype] * grad.abs() + 1e-37


def run_grad(x, token, g, ge, **kw):
    dev = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
    dev.copy_(x)
    _, h, _, _, m, ls = reference(x, token, 0)
    c = lambda t: None if t is None else t.float().cuda()
    got = M.logprobs_grad(dev, token.cuda() if g is not None else None, c(torch.stack([m, ls], 1)), c(h), c(g), c(ge), **kw)
    close(got, grad_reference(x, token, g, ge)[0], grad_bound(x, token, g, ge), "grad")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v", SIZES)
def test_grad_sizes(n, v, dtype):
    print(f"logprobs_grad n={n} v={v} {dtype}", flush=True)
    x, token = draw(n, v, dtype, n + v, masked=0.1 if v > 4 else 0.0)
    r = torch.Generator().manual_seed(n)
    g, ge = torch.randn(n, generator=r), torch.randn(n, generator=r)
    run_grad(x, token, g, ge)
    run_grad(x, token, g, None)
    run_grad(x, token, None, ge)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [64, 301, 5000])
def test_grad_rows_without_a_distribution(v, dtype):
    x = torch.randn(8, v, generator=torch.Generator().manual_seed(v)).to(dtype)
    x[1], x[2, 0], x[3, v - 1], x[4] = -INF, math.nan, INF, torch.finfo(dtype).min
    x[5, 1:] = -INF
    x[6] = math.nan
    token = torch.tensor([0, 1, 2, 3, 4, 0, -1, v], dtype=torch.int32)
    run_grad(x, token, torch.ones(8), None)                     # row 6: NaN, but it has no token: zeros
    run_grad(x, token, torch.ones(8), torch.tensor([0.0, 1, 0, 1, 0, 1, 0, 1]))
    run_grad(x, token, torch.zeros(8), torch.zeros(8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [64, 1001, 20000])
def test_grad_strides_and_in_place(v, dtype):
    for pad in (0, 1, 4, 8):
        x, token = draw(21, v, dtype, v + pad, pad=pad)
        g = torch.randn(21, generator=torch.Generator().manual_seed(1))
        print(f"logprobs_grad v={v} pad={pad} {dtype}", flush=True)
        run_grad(x, token, g, g)
        for opad in (0, 3, 8):
            wide = torch.full((21, v + opad), 7.0, dtype=dtype, device="cuda")
            run_grad(x, token, g, g, out=wide[:, :v])
            assert (wide[:, v:] == 7.0).all()
        wide = torch.full((21, v + pad), 7.0, dtype=dtype, device="cuda")
        y = wide[:, :v]
        y.copy_(x)
        fw = M.logprobs(y, token.cuda())
        got = M.logprobs_grad(y, token.cuda(), fw.stats, fw.entropy, g.cuda(), g.cuda(), out=y)
        assert got.data_ptr() == y.data_ptr() and (wide[:, v:] == 7.0).all()
        close(got, grad_reference(x, token, g, g)[0], grad_bound(x, token, g, g), "in place")


def test_grad_against_differences():
    """The kernels' gradient against central differences of the float64 definition (step 2^-12: off by
    about its square, 6e-8, times third derivatives of order 1)."""
    n, v, step = 6, 9, 2.0 ** -12
    x, _ = draw(n, v, torch.float32, 11, spread=1.5)
    token = torch.tensor([0, 3, 8, 5, -1, 1], dtype=torch.int32)
    r = torch.Generator().manual_seed(2)
    g, ge = torch.randn(n, generator=r).double(), torch.randn(n, generator=r).double()

    def loss(z):
        lp, h, *_ = reference(z, token, 0)
        return (g * lp + ge * h).sum()

    want = torch.zeros(n, v, dtype=torch.float64)
    for i in range(n):
        for j in range(v):
            e = torch.zeros(n, v, dtype=torch.float64)
            e[i, j] = step
            want[i, j] = (loss(x.double() + e) - loss(x.double() - e)) / (2 * step)
    fw = M.logprobs(x.cuda(), token.cuda())
    got = M.logprobs_grad(x.cuda(), token.cuda(), fw.stats, fw.entropy, g.float().cuda(), ge.float().cuda())
    assert (got.cpu().double() - want).abs().max() < 4e-6


# --- streams, graphs, refusals ------------------------------------------------------------------

def test_side_stream_and_graph():
    for n, v, k in ((500, 64, 4), (40, 3000, 8), (2, 70001, 5), (1, 300000, 16)):
        print(f"logprobs graph n={n} v={v}", flush=True)
        x, token = (t.cuda() for t in draw(n, v, torch.bfloat16, 21))
        g = torch.ones(n, device="cuda")
        want = M.logprobs(x, token, k=k)
        grad = M.logprobs_grad(x, token, want.stats, want.entropy, g, g)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        on_side = M.logprobs(x, token, k=k, stream=side)
        side.synchronize()
        for a, b in zip(on_side, want):
            assert torch.equal(a, b)
        need = max(16, M._train.load().maestro_logprobs_workspace(n, v, k, 1))
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        out = M.Logprobs(*[torch.empty_like(t) for t in want])
        gout = torch.empty_like(grad)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            M.logprobs(x, token, k=k, out=out, workspace=ws)
            M.logprobs_grad(x, token, out.stats, out.entropy, g, g, out=gout)
        for rep in range(3):
            for t in (*out, gout, ws):
                t.fill_(1)
            if rep == 1:
                M.logprobs(x, token, k=k)
                torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip((*out, gout), (*want, grad)):
                assert torch.equal(a, b), rep


def test_refusals():
    x = torch.zeros(4, 8, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    s, f = torch.zeros(4, 2, device="cuda"), torch.zeros(4, device="cuda")
    for bad, err in ((lambda: M.logprobs(x.half(), t), TypeError), (lambda: M.logprobs(x.cpu(), t), TypeError),
                     (lambda: M.logprobs(x.t(), t), ValueError), (lambda: M.logprobs(x[0], t), ValueError),
                     (lambda: M.logprobs(x, t.long()), TypeError), (lambda: M.logprobs(x, t[:3]), ValueError),
                     (lambda: M.logprobs(x, t, k=17), ValueError), (lambda: M.logprobs(x[:, :0], t), ValueError),
                     (lambda: M.logprobs(x[:1].expand(4, 8), t), ValueError),
                     (lambda: M.logprobs_grad(x, t, s, f, None), ValueError),
                     (lambda: M.logprobs_grad(x, t, s, None, f, f), ValueError),
                     (lambda: M.logprobs_grad(x, t, s[:3], f, f), ValueError),
                     (lambda: M.logprobs_grad(x, t, s, f, f, out=torch.zeros(4, 9, device="cuda")), ValueError),
                     (lambda: M.logprobs_grad(x, t, s, f, f, out=x.bfloat16()), ValueError)):
        with pytest.raises(err):
            bad()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v", [(450, 34), (3000, 3), (2500, 293), (1025, 9), (700, 505), (90, 520), (61, 2044), (21, 2049), (40, 4096)])
def test_grad_rows_end_to_end(n, v, dtype):
    """Workgroups that hold parts of rows, and both sides of the lines between the forms."""
    print(f"logprobs_grad n={n} v={v} {dtype}", flush=True)
    x, token = draw(n, v, dtype, n * v, masked=0.2 if v > 4 else 0.0, pad=3)
    r = torch.Generator().manual_seed(v)
    run_grad(x, token, torch.randn(n, generator=r), torch.randn(n, generator=r))


def test_grad_more_vectors_than_threads():
    n, v = 2_200_003, 7
    x, token = draw(n, v, torch.float32, 4)
    r = torch.Generator().manual_seed(9)
    run_grad(x, token, torch.randn(n, generator=r), torch.randn(n, generator=r))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [40, 3000, 20000])
def test_grad_of_masked_logits_with_large_coefficients(v, dtype):
    x, token = draw(12, v, dtype, v, masked=0.5)
    token.fill_(-1)
    ge = torch.full((12,), 1e30)
    run_grad(x, token, None, ge)
    dev = x.cuda()
    fw = M.logprobs(dev)
    got = M.logprobs_grad(dev, None, fw.stats, fw.entropy, None, ge.cuda())
    assert (got.cpu()[x == -INF] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v", [(5, 2047), (5, 2049), (2049, 4100), (2047, 4100), (2050, 20001), (3, 20481)])
def test_rows_by_a_wavefront_or_more(n, v, dtype):
    """Both sides of the lines between 64 and more threads for a row."""
    print(f"logprobs n={n} v={v} {dtype}", flush=True)
    check(*draw(n, v, dtype, n + 3 * v, masked=0.1), 6)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k", [0, 1, 2, 3, 4, 5])
@pytest.mark.parametrize("n,v", [(37, 513), (5, 700), (37, 1023), (9, 1025), (37, 1100), (9, 2047), (5, 2048)])
def test_rows_in_a_wavefronts_registers(n, v, k, dtype):
    print(f"logprobs n={n} v={v} k={k} {dtype}", flush=True)
    check(*draw(n, v, dtype, n + v + k, masked=0.2, pad=1), k)
    x, token = draw(n, v, dtype, n + v + k)
    x.copy_(x.round())                                          # ties
    x[0], x[1, :-1], x[2, v // 2], x[3, 1] = -INF, -INF, INF, math.nan
    check(x, token, k)
