"""maestro_layer and maestro_layer_grad against the products in float64 (on the CPU; large ones against
sampled rows and columns).

Bounds. Products of two bfloat16 are exact in float32, of two float32 off by 2^-24 of themselves; a sum of K
terms accumulated in float32 is off by at most K 2^-24 of the sum of magnitudes, and, as rounding errors have
no common sign, for long sums by a few times sqrt(K) 2^-24: 2^-24 (32 + 2 sqrt(K)) sum |a b| here. Outputs
in the layer's type are rounded once more, by at most 2^-9 (bfloat16) or 2^-24 of themselves."""
import math

import pytest
import torch

import paper_2606_12950_amd as M

pytestmark = pytest.mark.gpu
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def draw(n, i, o, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, i, generator=g)
    return (x.to(dtype), (torch.randn(o, i, generator=g) * i ** -0.5).to(dtype), torch.randn(o, generator=g),
            (torch.randn(n, o, generator=g) / max(n, 1)).to(dtype))


def bound(a, b):
    """of the product a b, both float64"""
    return 2.0 ** -24 * (32 + 2 * math.sqrt(a.shape[1])) * (a.abs() @ b.abs())


def near(got, want, tol, what):
    off = (got.cpu().double() - want).abs()
    wrong = ~(off <= tol)
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} off, first at {wrong.nonzero()[0].tolist()}, " \
        f"by up to {(off / tol.clamp_min(1e-300))[wrong].max():.3g} of the bound"


SIZES = [(1, 16, 16), (2, 32, 16), (15, 16, 48), (16, 64, 32), (17, 48, 80), (63, 64, 128), (64, 128, 32), (65, 272, 16),
         (100, 256, 64), (127, 16, 512), (128, 512, 512), (129, 144, 176), (255, 128, 256), (256, 256, 256), (257, 256, 272),
         (300, 256, 512), (511, 80, 1024), (1000, 1024, 64), (1, 1024, 1024), (31, 2048, 1040), (4096, 64, 128), (4096, 128, 32),
         (4099, 512, 64), (20011, 256, 512), (9000, 1024, 1024), (70001, 64, 48), (8, 16384, 32), (5, 32, 16384)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", SIZES)
def test_layer(n, i, o, dtype):
    print(f"layer n={n} {i}->{o} {dtype}", flush=True)
    x, w, b, _ = draw(n, i, o, dtype, n + i + o)
    xd, wd = x.double(), w.double()
    want = xd @ wd.t() + b.double()
    tol = bound(xd, wd.t()) + 2.0 ** -23 * b.double().abs() + ROUND[dtype] * want.abs()
    near(M.layer(x.cuda(), w.cuda(), b.cuda(), relu=False), want, tol, "z")
    y = M.layer(x.cuda(), w.cuda(), b.cuda(), relu=True)
    near(y, want.clamp_min(0), tol, "relu")
    assert (y >= 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", SIZES)
def test_layer_grad(n, i, o, dtype):
    print(f"layer_grad n={n} {i}->{o} {dtype}", flush=True)
    x, w, _, gz = draw(n, i, o, dtype, n + i + o + 1)
    x = torch.where(torch.rand(n, i, generator=torch.Generator().manual_seed(n)) < 0.2, 0.0, x).to(dtype)
    xd, wd, gd = x.double(), w.double(), gz.double()
    gx, gw, gb = gd @ wd, gd.t() @ xd, gd.sum(0)
    for relu, want_x in ((False, True), (True, True), (True, False)):
        got = M.layer_grad(x.cuda(), w.cuda(), gz.cuda(), relu_input=relu, want_x=want_x)
        near(got.weight, gw, bound(gd.t(), xd) + 1e-38, "weight")
        near(got.bias, gb, bound(gd.t(), torch.ones(n, 1, dtype=torch.float64))[:, 0] + 1e-38, "bias")
        assert (got.x is not None) == want_x
        if want_x:
            want = torch.where(xd > 0, gx, 0.0) if relu else gx
            near(got.x, want, bound(gd, wd) + ROUND[dtype] * want.abs(), "x")
            if relu:
                assert (got.x.cpu()[x <= 0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_empty_batch(dtype):
    x, w, b, gz = draw(0, 64, 32, dtype, 1)
    assert M.layer(x.cuda(), w.cuda(), b.cuda()).shape == (0, 32)
    got = M.layer_grad(x.cuda(), w.cuda(), gz.cuda())
    assert got.x.shape == (0, 64) and not got.weight.any() and not got.bias.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_do_not_see_each_other(dtype):
    """NaN and infinities in some rows stay in those rows of y and g_x; nothing past the last row is touched."""
    n, i, o = 200, 128, 96
    x, w, b, gz = draw(n, i, o, dtype, 5)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[[0, 63, 64, 130, n - 1]] = True
    for poison in (math.nan, math.inf):
        xp, gp = x.clone(), gz.clone()
        xp[bad, 3] = poison
        gp[bad, 5] = poison
        clean, dirty = (M.layer(t.cuda(), w.cuda(), b.cuda(), relu=False).cpu() for t in (x, xp))
        assert torch.equal(clean[~bad], dirty[~bad]) and not torch.isfinite(dirty[bad]).all(1).any()
        clean, dirty = (M.layer_grad(x.cuda(), w.cuda(), t.cuda()).x.cpu() for t in (gz, gp))
        assert torch.equal(clean[~bad], dirty[~bad]) and not torch.isfinite(dirty[bad]).all(1).any()
    buf = torch.full((n + 64, o), 7.0, dtype=dtype, device="cuda")
    M.layer(x.cuda(), w.cuda(), b.cuda(), out=buf[:n])
    assert (buf[n:] == 7.0).all()
    buf = torch.full((n + 64, i), 7.0, dtype=dtype, device="cuda")
    gw = torch.full((o + 8, i), 7.0, device="cuda")
    gb = torch.full((o + 8,), 7.0, device="cuda")
    M.layer_grad(x.cuda(), w.cuda(), gz.cuda(), out=M.LayerGrad(buf[:n], gw[:o], gb[:o]))
    assert (buf[n:] == 7.0).all() and (gw[o:] == 7.0).all() and (gb[o:] == 7.0).all()


def test_relu_of_nan_and_masked_inputs():
    """A NaN activation stays a NaN (it is not rectified away); a NaN input's place takes no gradient."""
    x, w, b, gz = (t.cuda() for t in draw(40, 32, 32, torch.bfloat16, 9))
    x[7, 2] = math.nan
    assert torch.isnan(M.layer(x, w, b, relu=True)[7]).all()
    assert M.layer_grad(x, w, gz, relu_input=True).x[7, 2] == 0


def test_offsets_past_32_bits():
    n, i, o = (1 << 22) + 5, 16, 528
    x = torch.randn(n, i, device="cuda").bfloat16()
    w = torch.randn(o, i, device="cuda").bfloat16()
    b = torch.zeros(o, device="cuda")
    y = M.layer(x, w, b, relu=False)
    at = torch.tensor([0, 1, 12345, n // 2, n - 65, n - 2, n - 1])
    xd, wd = x[at].cpu().double(), w.cpu().double()
    want = xd @ wd.t()
    near(y[at], want, bound(xd, wd.t()) + 2.0 ** -8 * want.abs(), "y")
    got = M.layer_grad(x, w, y, relu_input=False)
    yd = y[at].cpu().double()
    want = yd @ wd
    near(got.x[at], want, bound(yd, wd) + 2.0 ** -8 * want.abs(), "x")
    s = torch.zeros(o, i, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(s)
    for a in range(0, n, 1 << 18):
        g, xx = y[a:a + (1 << 18)].double(), x[a:a + (1 << 18)].double()
        s += torch.mm(g.t().contiguous(), xx)
        mag += torch.mm(g.abs().t().contiguous(), xx.abs())
    near(got.weight, s.cpu(), (2.0 ** -24 * (32 + 2 * math.sqrt(n)) * mag).cpu(), "weight")


def test_weight_gradient_against_differences():
    """d/dW of sum(G * (x W^T + b)): linear, so a difference quotient in float64 is exact but for rounding."""
    x, w, b, gz = draw(50, 32, 16, torch.float32, 13)
    got = M.layer_grad(x.cuda(), w.cuda(), gz.cuda(), relu_input=False)
    f = lambda ww, xx: (gz.double() * (xx @ ww.t() + b.double())).sum()
    for at in ((0, 0), (15, 31), (7, 16)):
        e = torch.zeros(16, 32, dtype=torch.float64)
        e[at] = 1.0
        d = (f(w.double() + e, x.double()) - f(w.double() - e, x.double())) / 2
        assert abs(got.weight[at].item() - d.item()) < 1e-6
    for at in ((0, 0), (49, 31), (20, 5)):
        e = torch.zeros(50, 32, dtype=torch.float64)
        e[at] = 1.0
        d = (f(w.double(), x.double() + e) - f(w.double(), x.double() - e)) / 2
        assert abs(got.x[at].item() - d.item()) < 1e-6


def test_graph_and_equal_bits():
    for n, i, o, dtype in ((3000, 256, 512, torch.bfloat16), (700, 64, 128, torch.float32), (90000, 128, 64, torch.bfloat16)):
        print(f"layers graph n={n} {i}->{o} {dtype}", flush=True)
        x, w, b, gz = (t.cuda() for t in draw(n, i, o, dtype, 3))
        want = (M.layer(x, w, b), *M.layer_grad(x, w, gz, relu_input=True))
        again = (M.layer(x, w, b), *M.layer_grad(x, w, gz, relu_input=True))
        for a, c in zip(again, want):
            assert torch.equal(a, c)
        ws = torch.empty(max(16, M._train.load().maestro_layer_grad_workspace(n, i, o, M._train._DTYPE[dtype])),
                         dtype=torch.uint8, device="cuda")
        y, out = torch.empty_like(want[0]), M.LayerGrad(*[torch.empty_like(t) for t in want[1:]])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            M.layer(x, w, b, out=y)
            M.layer_grad(x, w, gz, relu_input=True, out=out, workspace=ws)
        for rep in range(3):
            for t in (y, *out, ws):
                t.fill_(1)
            if rep == 1:
                M.layer_grad(x, w, gz)
                torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, c in zip((y, *out), want):
                assert torch.equal(a, c), rep


def test_refusals():
    x, w, b, gz = (t.cuda() for t in draw(8, 32, 16, torch.bfloat16, 1))
    for bad, err in ((lambda: M.layer(x.float(), w, b), TypeError), (lambda: M.layer(x, w, b.bfloat16()), TypeError),
                     (lambda: M.layer(x, w.half(), b), TypeError), (lambda: M.layer(x.cpu(), w, b), TypeError),
                     (lambda: M.layer(x[:, :16], w, b), ValueError), (lambda: M.layer(x, w, b[:8]), ValueError),
                     (lambda: M.layer(x, w, b, out=torch.empty(7, 16, dtype=x.dtype, device="cuda")), ValueError),
                     (lambda: M.layer(x[:, :24].contiguous(), w[:, :24].contiguous(), b), M.MaestroError),
                     (lambda: M.layer_grad(x, w, gz[:7]), ValueError),
                     (lambda: M.layer_grad(x, w, gz.float()), TypeError)):
        with pytest.raises(err):
            bad()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", [(338, 128, 128), (512, 32, 32), (513, 32, 32), (2000, 512, 512), (8192, 256, 64), (40000, 192, 192),
                                   (40001, 80, 160), (40000, 256, 144), (91341, 32, 48), (33000, 208, 256)])
def test_forms(n, i, o, dtype):
    """Both gradients in one launch or two, one or many shares of the rows, tiles that the widths do not fill."""
    print(f"forms n={n} {i}->{o} {dtype}", flush=True)
    x, w, b, gz = draw(n, i, o, dtype, n + 7 * i + o)
    xd, wd, gd = x.double(), w.double(), gz.double()
    z = xd @ wd.t() + b.double()
    near(M.layer(x.cuda(), w.cuda(), b.cuda(), relu=False), z,
         bound(xd, wd.t()) + 2.0 ** -23 * b.double().abs() + ROUND[dtype] * z.abs(), "z")
    gx = gd @ wd
    for want_x in (True, False):
        got = M.layer_grad(x.cuda(), w.cuda(), gz.cuda(), want_x=want_x)
        near(got.weight, gd.t() @ xd, bound(gd.t(), xd) + 1e-38, "weight")
        near(got.bias, gd.sum(0), bound(gd.t(), torch.ones(n, 1, dtype=torch.float64))[:, 0] + 1e-38, "bias")
        if want_x:
            near(got.x, gx, bound(gd, wd) + ROUND[dtype] * gx.abs(), "x")
