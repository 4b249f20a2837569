"""The layers by role, in 8-bit integers and from checkpoints as they are used: one after the other, on streams, replayed from a
graph, over arrays past 2^31 elements, and in a fit.

Bounds. Values that a definition gives are compared bit for bit. Gradients of weights: 2^-24 (32 + 2 sqrt(K)) sum |a b| for a sum
of K products in float32 (rounding errors have no common sign), once for each of the two sides compared."""
import math

import pytest
import torch

import paper_2606_12950_amd as M
from paper_2606_12950_amd import fit as F
from test_gpu_int8 import definition, quantized
from test_gpu_packed import packed, values

pytestmark = pytest.mark.gpu


def sums(a, b):
    """of the product a b in float32, both float64"""
    return 2.0 ** -24 * (32 + 2 * math.sqrt(a.shape[1])) * (a.abs() @ b.abs())


def near(got, want, tol):
    off = (got.double().cpu() - want.double().cpu()).abs()
    assert (off <= tol).all(), f"{int((~(off <= tol)).sum())} of {off.numel()} off, by up to {float((off / tol.clamp_min(1e-300)).max()):.3g} of the bound"


def test_served_in_8_bits():
    """Three layers, rows quantised between them, and the log probabilities: every stage as its definition has it."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(500, 256, generator=g).bfloat16()
    h, hd = x, x.cuda()
    for l, (i, o) in enumerate(((256, 512), (512, 512), (512, 64))):
        w, b = torch.randn(o, i, generator=g) * i ** -0.5, torch.randn(o, generator=g) * 0.1
        last = l == 2
        wq, wd = M.Quantized(*quantized(w)), M.quantize_rows(w.cuda())
        assert torch.equal(wd.codes.cpu(), wq.codes)
        dtype = torch.float32 if last else torch.bfloat16
        h = definition(M.Quantized(*quantized(h)), wq, b, not last, dtype)
        hd = M.layer_int8(M.quantize_rows(hd), wd, b.cuda(), relu=not last, dtype=dtype)
        assert torch.equal(hd.cpu(), h)
    bins = torch.randint(0, 64, (500,), generator=g, dtype=torch.int32)
    got = M.logprobs(hd, bins.cuda()).logprob.cpu().double()
    want = torch.log_softmax(h.double(), 1).gather(1, bins.long()[:, None])[:, 0]
    assert ((got - want).abs() <= 2.0 ** -18 * (1 + want.abs())).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_trained_by_role(dtype):
    """Roles' stages through networks of their own and back. Layers and input's gradients are bit for bit those of each role's rows
    alone; weights' gradients add the same products, in another order."""
    sizes, dims = [300, 0, 1, 77, 640], (64, 128, 32)
    n, groups = sum(sizes), len(sizes)
    ends = [0]
    for s in sizes:
        ends.append(ends[-1] + s)
    off = torch.tensor(ends, device="cuda")
    g = torch.Generator().manual_seed(3)
    x = torch.randn(n, dims[0], generator=g).to(dtype).cuda()
    ws = [(torch.randn(groups, o, i, generator=g) * i ** -0.5).to(dtype).cuda() for i, o in zip(dims, dims[1:])]
    bs = [(torch.randn(groups, o, generator=g) * 0.1).cuda() for o in dims[1:]]
    bins = torch.randint(0, dims[-1], (n,), generator=g, dtype=torch.int32).cuda()
    h = M.layer_grouped(x, ws[0], bs[0], off)
    z = M.layer_grouped(h, ws[1], bs[1], off, relu=False)
    s = M.logprobs(z, bins)
    gz = M.logprobs_grad(z, bins, s.stats, s.entropy, torch.full((n,), -1.0 / n, device="cuda"))
    g1 = M.layer_grouped_grad(h, ws[1], gz, off, relu_input=True)
    g0 = M.layer_grouped_grad(x, ws[0], g1.x, off, want_x=False)
    for r, (a, b) in enumerate(zip(ends, ends[1:])):
        assert torch.equal(h[a:b], M.layer(x[a:b], ws[0][r], bs[0][r]))
        assert torch.equal(z[a:b], M.layer(h[a:b], ws[1][r], bs[1][r], relu=False))
        alone = M.layer_grad(h[a:b], ws[1][r], gz[a:b], relu_input=True)
        assert torch.equal(g1.x[a:b], alone.x)
        for got, inp, out in ((g1, h, gz), (g0, x, g1.x)):
            od, xd = out[a:b].double().cpu(), inp[a:b].double().cpu()
            near(got.weight[r], od.t() @ xd, sums(od.t(), xd) + 1e-38)
            near(got.bias[r], od.sum(0), sums(od.t(), torch.ones(b - a, 1, dtype=torch.float64))[:, 0] + 1e-38)
    grads = [g0.weight, g0.bias, g1.weight, g1.bias]
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    assert abs(float(M.clip_gradients(grads, norm / 2)) - norm) <= 2.0 ** -22 * norm


def calls(dtype, n=700, i=256, o=192):
    """Every operator on inputs that refill() writes anew: (refill, run); run returns all outputs."""
    g = torch.Generator().manual_seed(9)
    x, gz = torch.empty(n, i, dtype=dtype, device="cuda"), torch.empty(n, o, dtype=dtype, device="cuda")
    wg = (torch.randn(3, o, i, generator=g) * i ** -0.5).to(dtype).cuda()
    b, wq = torch.randn(3, o, generator=g).cuda(), M.quantize_rows(wg[0].contiguous())
    off = torch.zeros(4, dtype=torch.int64, device="cuda")

    def refill(seed):
        r = torch.Generator().manual_seed(seed)
        x.copy_(torch.randn(n, i, generator=r).relu_())
        gz.copy_(torch.randn(n, o, generator=r) / n)
        cuts = torch.randint(0, n + 1, (2,), generator=r).sort().values.tolist()
        off.copy_(torch.tensor([0, *cuts, n]))

    def run():
        q = M.quantize_rows(x)
        p, f = M.pack_activations(x, rectified=True), M.pack_activations(x)
        return [M.layer_grouped(x, wg, b, off), *M.layer_grouped_grad(x, wg, gz, off, relu_input=True), q.codes, q.scale,
                M.layer_int8(q, wq, b[0], dtype=dtype), p.codes, p.exponents, M.unpack_activations(p, dtype=dtype),
                *M.layer_grad_packed(p, wg[0], gz, relu_input=True), *M.layer_grad_packed(f, wg[0], gz)]
    return refill, run


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_replayed_from_a_graph(dtype):
    """Replays over other inputs, other group sizes too, with eager calls and synchronisations between them."""
    refill, run = calls(dtype)
    refill(0)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in range(1, 6):
        refill(seed)
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        eager = run()
        assert all(torch.equal(a, z) for a, z in zip(kept, eager)), seed


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_two_streams_at_once(dtype):
    """The same calls on two streams side by side, each with inputs of its own."""
    pairs = [calls(dtype), calls(dtype, n=1501, i=128, o=512)]
    want = []
    for k, (refill, run) in enumerate(pairs):
        refill(k)
        want.append(run())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    got = [[] for _ in pairs]
    for _ in range(4):
        for k, (_, run) in enumerate(pairs):
            with torch.cuda.stream(streams[k]):
                got[k].append(run())
    torch.cuda.synchronize()
    for k in range(2):
        for outs in got[k]:
            assert all(torch.equal(a, z) for a, z in zip(outs, want[k]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_stream_and_out_arguments(dtype):
    """An explicit stream, and outputs and workspaces of the caller's, give what plain calls give."""
    n, i, o = 300, 64, 48
    g = torch.Generator().manual_seed(2)
    x, gz = torch.randn(n, i, generator=g).to(dtype).cuda(), torch.randn(n, o, generator=g).to(dtype).cuda()
    w, b = torch.randn(2, o, i, generator=g).to(dtype).cuda(), torch.randn(2, o, generator=g).cuda()
    off = torch.tensor([0, 111, 300], device="cuda")
    wq, q, p = M.quantize_rows(w[0].contiguous()), M.quantize_rows(x), M.pack_activations(x)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    e = lambda *s, t=dtype: torch.empty(s, dtype=t, device="cuda")
    grad = lambda *lead: M.LayerGrad(e(n, i), e(*lead, o, i, t=torch.float32), e(*lead, o, t=torch.float32))
    plain = [M.layer_grouped(x, w, b, off), *M.layer_grouped_grad(x, w, gz, off), *q, M.layer_int8(q, wq, b[0], dtype=dtype), *p,
             M.unpack_activations(p, dtype=dtype), *M.layer_grad_packed(p, w[0], gz)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    by_stream = [M.layer_grouped(x, w, b, off, stream=s), *M.layer_grouped_grad(x, w, gz, off, stream=s), *M.quantize_rows(x, stream=s),
                 M.layer_int8(q, wq, b[0], dtype=dtype, stream=s), *M.pack_activations(x, stream=s),
                 M.unpack_activations(p, dtype=dtype, stream=s), *M.layer_grad_packed(p, w[0], gz, stream=s)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, z) for a, z in zip(plain, by_stream))
    by_out = [M.layer_grouped(x, w, b, off, out=e(n, o)), *M.layer_grouped_grad(x, w, gz, off, out=grad(2), workspace=ws),
              *M.quantize_rows(x, out=M.Quantized(e(n, i, t=torch.int8), e(n, t=torch.float32))),
              M.layer_int8(q, wq, b[0], dtype=dtype, out=e(n, o)),
              *M.pack_activations(x, out=M.Packed(e(n, i, t=torch.int8), e(n, 2, t=torch.uint8))),
              M.unpack_activations(p, dtype=dtype, out=e(n, i)), *M.layer_grad_packed(p, w[0], gz, out=grad(), workspace=ws)]
    assert all(torch.equal(a, z) for a, z in zip(plain, by_out))
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(M.MaestroError, match="workspace too small"):
        M.layer_grouped_grad(torch.cat([x] * 9), w, torch.cat([gz] * 9), off, workspace=small)


def test_unaligned_and_strided_are_refused():
    flat = torch.randn(64 * 32 + 8, device="cuda")
    at4 = flat[1:64 * 32 + 1].view(64, 32)                    # rows of float32 that begin 4 bytes past 16
    for call in (lambda: M.quantize_rows(at4), lambda: M.pack_activations(at4),
                 lambda: M.layer_grouped(at4, torch.zeros(1, 16, 32, device="cuda"), torch.zeros(1, 16, device="cuda"),
                                         torch.tensor([0, 64], device="cuda"))):
        with pytest.raises(M.MaestroError, match="invalid argument"):
            call()
    wide = torch.randn(64, 64, device="cuda")[:, :32]
    for call in (lambda: M.quantize_rows(wide), lambda: M.pack_activations(wide)):
        with pytest.raises(ValueError, match="contiguous"):
            call()
    with pytest.raises(M.MaestroError, match="unsupported"):
        M.quantize_rows(torch.randn(4, 24, device="cuda"))
    # a scale and exponents may begin anywhere
    x = torch.randn(64, 32, device="cuda")
    scale, exponents = torch.empty(65, device="cuda")[1:], torch.empty(65, 1, dtype=torch.uint8, device="cuda")[1:]
    q = M.quantize_rows(x, out=M.Quantized(torch.empty(64, 32, dtype=torch.int8, device="cuda"), scale))
    p = M.pack_activations(x, out=M.Packed(torch.empty(64, 32, dtype=torch.int8, device="cuda"), exponents))
    assert torch.equal(q.scale, M.quantize_rows(x).scale) and torch.equal(p.exponents, M.pack_activations(x).exponents)
    w, gz = torch.randn(16, 32, device="cuda"), torch.randn(64, 16, device="cuda")
    assert all(torch.equal(a, z) for a, z in zip(M.layer_grad_packed(p, w, gz), M.layer_grad_packed(M.pack_activations(x), w, gz)))
    assert torch.equal(M.unpack_activations(p), M.unpack_activations(M.pack_activations(x)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_arrays_past_32_bits(dtype):
    """2^21 + 77 rows of 1,040 values (2.2 * 10^9 elements): the last rows are those of a call on them alone."""
    n, d, o, tail = (1 << 21) + 77, 1040, 16, 1000
    x = torch.zeros(n, d, dtype=dtype, device="cuda")
    g = torch.Generator().manual_seed(7)
    x[-tail:] = torch.randn(tail, d, generator=g).to(dtype).cuda()
    end = x[-tail:].contiguous()
    q, qe = M.quantize_rows(x), M.quantize_rows(end)
    assert torch.equal(q.codes[-tail:], qe.codes) and torch.equal(q.scale[-tail:], qe.scale) and not q.codes[:1000].any()
    w = M.quantize_rows(torch.randn(o, d, generator=g).cuda())
    b = torch.randn(o, generator=g).cuda()
    assert torch.equal(M.layer_int8(q, w, b, dtype=dtype)[-tail:], M.layer_int8(qe, w, b, dtype=dtype))
    # outputs past 32 bits: 16 -> 1,040
    qx = M.Quantized(q.codes[:, :16].contiguous(), q.scale)
    wide = M.quantize_rows(torch.randn(d, 16, generator=g).cuda())
    bw = torch.randn(d, generator=g).cuda()
    y = M.layer_int8(qx, wide, bw, dtype=dtype)
    assert torch.equal(y[-tail:], M.layer_int8(M.Quantized(qx.codes[-tail:].contiguous(), q.scale[-tail:].contiguous()), wide, bw, dtype=dtype))
    del y, q, qx
    p, pe = M.pack_activations(x), M.pack_activations(end)
    assert torch.equal(p.codes[-tail:], pe.codes) and torch.equal(p.exponents[-tail:], pe.exponents)
    assert torch.equal(M.unpack_activations(p, dtype=dtype)[-tail:], M.unpack_activations(pe, dtype=dtype))
    # rows of zeros add nothing to the weights' gradient
    wt = torch.randn(o, d, generator=g).to(dtype).cuda()
    gz = torch.randn(n, o, generator=g).to(dtype).cuda()
    v, gd = values(*(t.cpu() for t in pe)), gz[-tail:].double().cpu()
    got = M.layer_grad_packed(p, wt, gz)
    near(got.weight, gd.t() @ v, sums(gd.t(), v))
    assert torch.equal(got.x[-tail:], M.layer_grad_packed(pe, wt, gz[-tail:].contiguous()).x)
    del p
    off = torch.tensor([0, 5, n - 300, n], device="cuda")
    wg = torch.stack([wt, 2 * wt, 3 * wt])
    bg = torch.randn(3, o, generator=g).cuda()
    y = M.layer_grouped(x, wg, bg, off, relu=False)
    assert torch.equal(y[-300:], M.layer(end[-300:].contiguous(), wg[2], bg[2], relu=False))
    assert torch.equal(y[-tail:-300], M.layer(end[:-300].contiguous(), wg[1], bg[1], relu=False))
    got = M.layer_grouped_grad(x, wg, gz, off)
    xd = end.double().cpu()
    near(got.weight[2], gd[-300:].t() @ xd[-300:], sums(gd[-300:].t(), xd[-300:]))
    near(got.weight[1], gd[:-300].t() @ xd[:-300], sums(gd[:-300].t(), xd[:-300]))
    assert torch.equal(got.x[-300:], M.layer_grad(end[-300:].contiguous(), wg[2], gz[-300:].contiguous()).x)


def network(dims, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return ([(torch.randn(o, i, generator=g) * i ** -0.5).to(dtype).cuda() for i, o in zip(dims[:-1], dims[1:])],
            [(torch.randn(o, generator=g) * 0.1).cuda() for o in dims[1:]])


@pytest.mark.parametrize("dims,dtype,n", [((64, 128, 32), torch.float32, 300), ((256, 512, 512, 64), torch.bfloat16, 1001),
                                          ((16, 48, 80, 32, 16), torch.bfloat16, 77), ((32, 16), torch.float32, 5)])
def test_fit_from_checkpoints(dims, dtype, n):
    """A Fit that keeps 8 bits has the same likelihoods, and the gradients of the layers with the kept values as their inputs."""
    x = torch.randn(n, dims[0], generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    bins = torch.randint(0, dims[-1], (n,), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    plain, kept = F.Fit(*network(dims, dtype, 5), n), F.Fit(*network(dims, dtype, 5), n, packed=True)
    assert torch.equal(plain.score(x, bins).logprob, kept.score(x, bins).logprob)
    hidden = [values(*packed(h.float().cpu(), True)) for h in plain.hidden[:-1]]
    for p, want in zip(kept.kept, hidden):
        assert torch.equal(M.unpack_activations(p, dtype=dtype).double().cpu(), want)
    plain.gradients(x, bins)
    gw, gb = kept.gradients(x, bins)
    g = M.logprobs_grad(plain.hidden[-1], bins, plain.out.stats, plain.out.entropy, torch.full((n,), -1.0 / n, device="cuda"))
    for l in reversed(range(len(dims) - 1)):
        v = (hidden[l - 1].to(dtype).cuda() if l else x)
        want = M.layer_grad(v, plain.weights[l], g, relu_input=l > 0, want_x=l > 0)
        gd, vd = g.double().cpu(), v.double().cpu()
        near(gw[l], want.weight, 2 * sums(gd.t(), vd) + 1e-38)
        near(gb[l], want.bias, 2 * sums(gd.t(), torch.ones(n, 1, dtype=torch.float64))[:, 0] + 1e-38)
        g = want.x
    mean, norm = kept.step(x, bins, 0.1)
    assert math.isfinite(float(mean)) and math.isfinite(float(norm)) and all(torch.isfinite(w).all() for w in kept.weights)


def test_the_command_keeps_8_bits():
    assert F.main(["--workload", "c1", "--stages", "2048", "--steps", "2", "--packed"])["stages"] == 2048


def test_a_fit_from_checkpoints_replays_from_a_graph():
    dims, n = (256, 512, 512, 64), 3001
    g = torch.Generator().manual_seed(6)
    x = torch.randn(n, 256, generator=g).bfloat16().cuda()
    bins = torch.randint(0, 64, (n,), generator=g, dtype=torch.int32).cuda()
    f = F.Fit(*network(dims, torch.bfloat16, 1), n, packed=True)

    def run():
        f.score(x, bins)
        f.gradients(x, bins)
        M.clip_gradients([*f.g_weights, *f.g_biases], 0.5, norm=f.norm, workspace=f.workspace)

    run()
    torch.cuda.synchronize()
    outs = (*f.g_weights, *f.g_biases, f.norm, f.out.logprob)
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(3):
        for t in (*outs, f.workspace, *(k for p in f.kept for k in p), *f.hidden):
            t.fill_(3)
        if rep == 1:
            f.score(x, bins)
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_a_fit_from_checkpoints_holds_less():
    """Bytes of a Fit's layers, plain and with the hidden ones kept in 8 bits: one buffer for the values of one hidden layer, two for
    more, a byte a value kept and one for every 32."""
    n = 40000
    for dims, dtype in (((64, 128, 32), torch.float32), ((256, 512, 64), torch.bfloat16), ((256, 512, 512, 64), torch.bfloat16),
                        ((16, 48, 80, 32, 16), torch.bfloat16), ((32, 16), torch.float32)):
        size, hidden = torch.finfo(dtype).bits // 8, dims[1:-1]
        held = {}
        for kept in (False, True):
            w, b = network(dims, dtype, 5)
            f = F.Fit(w, b, n, packed=kept)
            tensors = [*f.hidden, *f.g_z, *(t for p in f.kept or () for t in p)]
            held[kept] = sum({t.untyped_storage().data_ptr(): t.untyped_storage().nbytes() for t in tensors}.values())
        logits = 2 * n * size * dims[-1]
        buffers = min(2, len(hidden)) * n * size * max(hidden, default=0)
        assert held[False] == logits + 2 * n * size * sum(hidden), (dims, held)
        assert held[True] == logits + buffers + n * sum(h + -(-h // 32) for h in hidden), (dims, held)
        assert held[True] < held[False] or not hidden, (dims, held)
