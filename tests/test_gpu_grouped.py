"""maestro_layer_grouped and maestro_layer_grouped_grad against every group's products in float64 on the CPU.

Bounds, as for a layer of one group. Products of two bfloat16 are exact in float32, of two float32 off by 2^-24 of
themselves; a sum of K terms accumulated in float32 is off by at most K 2^-24 of the sum of magnitudes and, as rounding
errors have no common sign, for long sums by a few times sqrt(K) 2^-24: 2^-24 (32 + 2 sqrt(K)) sum |a b| here. Outputs in
the layer's type are rounded once more, by at most 2^-8 (bfloat16) or 2^-24 (float32, doubled here) of themselves."""
import math

import pytest
import torch

import paper_2606_12950_amd as M

pytestmark = pytest.mark.gpu
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def draw(n, groups, i, o, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, i, generator=g).to(dtype), (torch.randn(groups, o, i, generator=g) * i ** -0.5).to(dtype),
            torch.randn(groups, o, generator=g), (torch.randn(n, o, generator=g) / max(n, 1)).to(dtype))


def bound(a, b):
    """of the product a b, both float64"""
    return 2.0 ** -24 * (32 + 2 * math.sqrt(a.shape[1])) * (a.abs() @ b.abs())


def near(got, want, tol, what):
    off = (got.cpu().double() - want).abs()
    wrong = ~(off <= tol)
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} off, first at {wrong.nonzero()[0].tolist()}, " \
        f"by up to {(off / tol.clamp_min(1e-300))[wrong].max():.3g} of the bound"


def ranges(offsets, n):
    """[first, last) of every group: an offset below an earlier one counts as that one, one outside 0 .. n as the nearer bound."""
    most, out = 0, []
    for v in offsets:
        most = max(most, min(max(v, 0), n))
        out.append(most)
    return list(zip(out, out[1:]))


def check(offsets, n, i, o, dtype, seed=0):
    groups = len(offsets) - 1
    print(f"grouped n={n} {i}->{o} {dtype} offsets {offsets[:20]}", flush=True)
    x, w, b, gz = draw(n, groups, i, o, dtype, seed + n + i + o)
    x = torch.where(torch.rand(n, i, generator=torch.Generator().manual_seed(n)) < 0.2, 0.0, x).to(dtype)
    off = torch.tensor(offsets, dtype=torch.int64, device="cuda")
    xc, wc, bc, gc = x.cuda(), w.cuda(), b.cuda(), gz.cuda()
    y = {r: M.layer_grouped(xc, wc, bc, off, relu=r, out=torch.full((n, o), 7.0, dtype=dtype, device="cuda")) for r in (False, True)}
    grads = {}
    for relu, want_x in ((False, True), (True, True), (True, False)):
        out = M.LayerGrad(torch.full((n, i), 7.0, dtype=dtype, device="cuda") if want_x else None,
                          torch.full((groups, o, i), 7.0, device="cuda"), torch.full((groups, o), 7.0, device="cuda"))
        grads[relu, want_x] = M.layer_grouped_grad(xc, wc, gc, off, relu_input=relu, want_x=want_x, out=out)
    taken = torch.zeros(n, dtype=torch.bool)
    for g, (a, z) in enumerate(ranges(offsets, n)):
        taken[a:z] = True
        xd, wd, gd = x[a:z].double(), w[g].double(), gz[a:z].double()
        want = xd @ wd.t() + b[g].double()
        tol = bound(xd, wd.t()) + 2.0 ** -23 * b[g].double().abs() + ROUND[dtype] * want.abs()
        near(y[False][a:z], want, tol, f"z of group {g}")
        near(y[True][a:z], want.clamp_min(0), tol, f"y of group {g}")
        gx, gw, gb = gd @ wd, gd.t() @ xd, gd.sum(0)
        for (relu, want_x), got in grads.items():
            near(got.weight[g], gw, bound(gd.t(), xd) + 1e-38, f"weights of group {g}")
            near(got.bias[g], gb, bound(gd.t(), torch.ones(z - a, 1, dtype=torch.float64))[:, 0] + 1e-38, f"biases of group {g}")
            if want_x:
                v = torch.where(xd > 0, gx, 0.0) if relu else gx
                near(got.x[a:z], v, bound(gd, wd) + ROUND[dtype] * v.abs(), f"x of group {g}")
    # rows of no group are as they were
    for t in (y[False], y[True], grads[False, True].x, grads[True, True].x):
        assert (t[~taken.cuda()] == 7.0).all()


def offsets_of(sizes, first=0):
    out = [first]
    for s in sizes:
        out.append(out[-1] + s)
    return out


CASES = [([1], 16, 16), ([0, 1, 0], 16, 32), ([3, 0, 5, 1], 48, 80), ([15, 16, 17], 64, 128), ([63, 64, 65, 0], 32, 48),
         ([127, 128, 129], 144, 64), ([1] * 70, 80, 16), ([0] * 100 + [200] + [0] * 155, 64, 64), ([300, 0, 1, 255], 256, 512),
         ([1000, 3], 512, 64), ([2, 5, 700], 16, 1024), ([33] * 256, 16, 48), ([4096], 272, 144), ([1, 1], 1024, 1024),
         ([5000, 1, 0, 9000], 128, 256), ([3000, 4000], 1024, 96), ([100, 0, 200, 0], 4096, 2048)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,i,o", CASES)
def test_groups(sizes, i, o, dtype):
    check(offsets_of(sizes), sum(sizes), i, o, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,i,o", [([41000, 3, 30000], 192, 256), ([50001, 0, 90002], 256, 272), ([2, 140000], 64, 160),
                                       ([900, 0, 901] * 75, 256, 272)])
def test_many_rows(sizes, i, o, dtype):
    """The larger tiles, and groups of many shares next to groups of one."""
    check(offsets_of(sizes), sum(sizes), i, o, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_no_group(dtype):
    check(offsets_of([20, 0, 100], 37), 200, 64, 48, dtype)
    check(offsets_of([0, 0], 5), 12, 64, 48, dtype)          # none in any
    check(offsets_of([600, 700], 100), 1500, 256, 256, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offsets", [[0, 50, 30, 100], [-5, 20, 400, 900], [90, 10, 20], [1 << 40, 0, -(1 << 60)], [0, 1 << 62, 7, 100]])
def test_offsets_out_of_order(offsets, dtype):
    check(offsets, 150, 32, 64, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_rows(dtype):
    x, w, b, gz = draw(0, 3, 64, 32, dtype, 1)
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    assert M.layer_grouped(x.cuda(), w.cuda(), b.cuda(), off).shape == (0, 32)
    got = M.layer_grouped_grad(x.cuda(), w.cuda(), gz.cuda(), off)
    assert got.x.shape == (0, 64) and got.weight.shape == (3, 32, 64) and not got.weight.any() and not got.bias.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_group_is_a_layer(dtype):
    """Bit for bit: the sums of a tile are the same ones."""
    x, w, b, _ = draw(5000, 1, 256, 128, dtype, 3)
    off = torch.tensor([0, 5000], device="cuda")
    assert torch.equal(M.layer_grouped(x.cuda(), w.cuda(), b.cuda(), off), M.layer(x.cuda(), w[0].cuda(), b[0].cuda()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_groups_do_not_see_each_other(dtype):
    """NaN and infinities stay in their rows of y and g_x, and in their group's weights' and biases' gradients."""
    sizes, i, o = [70, 65, 1, 200], 64, 96
    n, off = sum(sizes), torch.tensor(offsets_of(sizes), device="cuda")
    x, w, b, gz = draw(n, 4, i, o, dtype, 5)
    for poison in (math.nan, math.inf):
        xp, gp = x.clone(), gz.clone()
        xp[100, 3] = poison          # of group 1
        gp[100, 5] = poison
        clean, dirty = (M.layer_grouped(t.cuda(), w.cuda(), b.cuda(), off, relu=False).cpu() for t in (x, xp))
        rest = torch.arange(n) != 100
        assert torch.equal(clean[rest], dirty[rest]) and not torch.isfinite(dirty[100]).all()
        a = M.layer_grouped_grad(x.cuda(), w.cuda(), gz.cuda(), off)
        z = M.layer_grouped_grad(xp.cuda(), w.cuda(), gp.cuda(), off)
        others = [0, 2, 3]
        assert torch.equal(a.x.cpu()[rest], z.x.cpu()[rest])
        assert torch.equal(a.weight[others], z.weight[others]) and torch.equal(a.bias[others], z.bias[others])
        assert not torch.isfinite(z.weight[1]).all() and not torch.isfinite(z.bias[1]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,i,o", [([3, 41000, 0, 30077], 272, 272), ([130000, 5, 10001], 528, 272), ([500, 1500, 7], 272, 80),
                                       ([20001, 33, 19000], 48, 176)])
def test_poison_in_large_groups(sizes, i, o, dtype):
    """As above in the larger tiles and shares; rows of no group before and behind hold NaN, as does the workspace."""
    ends = offsets_of(sizes, 9)
    n, groups = ends[-1] + 70, len(sizes)
    off = torch.tensor(ends, device="cuda")
    x, w, b, gz = (t.cuda() for t in draw(n, groups, i, o, dtype, 6))
    clean, grads = M.layer_grouped(x, w, b, off, relu=False), M.layer_grouped_grad(x, w, gz, off)
    for t in (x, gz):
        t[:9], t[ends[-1]:] = math.nan, math.nan
    taken = slice(9, ends[-1])
    ws = torch.full((1 << 28,), 0xFF, dtype=torch.uint8, device="cuda")
    again = M.layer_grouped_grad(x, w, gz, off, workspace=ws)
    assert torch.equal(M.layer_grouped(x, w, b, off, relu=False)[taken], clean[taken]) and torch.equal(again.x[taken], grads.x[taken])
    assert torch.equal(again.weight, grads.weight) and torch.equal(again.bias, grads.bias)
    bad = [9, ends[1], (ends[1] + ends[2]) // 2, ends[2] - 1]               # the first row of the first group, and three of the second
    x[bad, i - 1] = math.nan
    gz[bad, o - 1] = math.inf
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[bad], rest[:9], rest[ends[-1]:] = False, False, False
    assert torch.equal(M.layer_grouped(x, w, b, off, relu=False)[rest], clean[rest])
    dirty = M.layer_grouped_grad(x, w, gz, off, workspace=ws)
    assert torch.equal(dirty.x[rest], grads.x[rest])
    others = list(range(2, groups))
    assert torch.equal(dirty.weight[others], grads.weight[others]) and torch.equal(dirty.bias[others], grads.bias[others])
    for g in (0, 1):
        assert torch.equal(dirty.weight[g, :-1, :-1], grads.weight[g, :-1, :-1]) and torch.equal(dirty.bias[g, :-1], grads.bias[g, :-1])
        assert torch.isnan(dirty.weight[g, :, -1]).all() and torch.isinf(dirty.bias[g, -1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_calls_and_nothing_beside(dtype):
    sizes, i, o = [700, 0, 900], 256, 192
    n, off = sum(sizes), torch.tensor(offsets_of(sizes), device="cuda")
    x, w, b, gz = (t.cuda() for t in draw(n, 3, i, o, dtype, 9))
    first = M.layer_grouped_grad(x, w, gz, off)
    bx = torch.full((n + 8, i), 7.0, dtype=dtype, device="cuda")
    bw, bb = torch.full((4, o, i), 7.0, device="cuda"), torch.full((4, o), 7.0, device="cuda")
    again = M.layer_grouped_grad(x, w, gz, off, out=M.LayerGrad(bx[:n], bw[:3], bb[:3]))
    assert all(torch.equal(a, z) for a, z in zip(first, again))
    assert (bx[n:] == 7.0).all() and (bw[3] == 7.0).all() and (bb[3] == 7.0).all()
    by = torch.full((n + 8, o), 7.0, dtype=dtype, device="cuda")
    assert torch.equal(M.layer_grouped(x, w, b, off), M.layer_grouped(x, w, b, off, out=by[:n])) and (by[n:] == 7.0).all()


def test_gradient_is_the_difference():
    """g_x, g_w and g_b against central differences of the float32 layer's own outputs, in float64 sums: a step h changes the
    output linearly, so only the outputs' rounding remains, 2^-22 of their size over 2 h."""
    sizes, i, o = [5, 0, 9], 16, 16
    n, off = sum(sizes), torch.tensor(offsets_of(sizes), device="cuda")
    x, w, b, gz = (t.cuda() for t in draw(n, 3, i, o, torch.float32, 11))
    got = M.layer_grouped_grad(x, w, gz, off)
    h = 0.25
    loss = lambda x, w, b: (M.layer_grouped(x, w, b, off, relu=False).double() * gz.double()).sum()
    size = float((M.layer_grouped(x, w, b, off, relu=False).double().abs() * gz.double().abs()).sum()) + 1.0
    tol = 2.0 ** -22 * 8 * size / (2 * h)
    for t, grad in ((x, got.x), (w, got.weight), (b, got.bias)):
        for at in [0, 7, t.numel() // 2, t.numel() - 1]:
            shifted = []
            for s in (h, -h):
                p = t.clone()
                p.view(-1)[at] += s
                shifted.append(loss(*(p if u is t else u for u in (x, w, b))))
            assert abs(float((shifted[0] - shifted[1]) / (2 * h)) - float(grad.reshape(-1)[at])) <= tol
