"""The layers by role, from kept bytes and in 8-bit integers at the sizes of every one of their kernels (layer_forms), against float64 on the
GPU in blocks of rows. Bounds as in test_gpu_grouped: 2^-24 (32 + 2 sqrt(K)) sum |a b| for a sum of K products, and one rounding of
outputs in the layer's type. Whole numbers bit for bit."""
import math

import pytest
import torch

import paper_2606_12950_amd as M
from paper_2606_12950_amd import _layers
from layer_forms import GROUPED, INT8, PACKED

pytestmark = pytest.mark.gpu
ROWS = 1 << 14
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def near(got, want, tol, what):
    off = (got.double() - want).abs()
    wrong = ~(off <= tol)
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} off, first at {wrong.nonzero()[0].tolist()}, " \
        f"by up to {(off / tol.clamp_min(1e-300))[wrong].max():.3g} of the bound"


def sums(k):
    return 2.0 ** -24 * (32 + 2 * math.sqrt(k))


def weights_grad(gz, x):
    """(g_w, its sum of magnitudes, g_b, its sum of magnitudes) in float64; x gives rows a .. z."""
    o = gz.shape[1]
    gw = mw = 0.0
    gb, mb = (torch.zeros(o, dtype=torch.float64, device="cuda") for _ in range(2))
    for a in range(0, gz.shape[0], ROWS):
        g, v = gz[a:a + ROWS].double(), x(a, min(a + ROWS, gz.shape[0]))
        gt = g.t().contiguous()
        gw, mw = gw + torch.mm(gt, v), mw + torch.mm(gt.abs(), v.abs())
        gb, mb = gb + g.sum(0), mb + g.abs().sum(0)
    return gw, mw, gb, mb


def check_weights(got_w, got_b, gz, x, what):
    gw, mw, gb, mb = weights_grad(gz, x)
    near(got_w, gw, sums(gz.shape[0]) * mw + 1e-38, f"weights {what}")
    near(got_b, gb, sums(gz.shape[0]) * mb + 1e-38, f"biases {what}")


def check_input(got, gz, w, positive, dtype, what):
    wd = w.double()
    for a in range(0, gz.shape[0], ROWS):
        g = gz[a:a + ROWS].double()
        want, size = torch.mm(g, wd), torch.mm(g.abs(), wd.abs())
        if positive is not None:
            want = torch.where(positive(a, a + ROWS), want, 0.0)
        near(got[a:a + ROWS], want, sums(gz.shape[1]) * size + ROUND[dtype] * want.abs(), f"x {what}, rows from {a}")


def inputs(n, groups, i, o, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = torch.where(torch.rand(n, i, generator=g, device="cuda") < 0.2, 0.0, r(n, i)).to(dtype)
    return x, (r(groups, o, i) * i ** -0.5).to(dtype), r(groups, o), (r(n, o) / n).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,i,o", GROUPED)
def test_grouped(sizes, i, o, dtype):
    n, groups = sum(sizes), len(sizes)
    print(f"grouped n={n} in {groups} {i}->{o} {dtype}", flush=True)
    ends = [3]                                                # rows of no group before and behind
    for s in sizes:
        ends.append(ends[-1] + s)
    rows = ends[-1] + 5
    x, w, b, gz = inputs(rows, groups, i, o, dtype, n + i + o)
    off = torch.tensor(ends, device="cuda")
    y = M.layer_grouped(x, w, b, off, out=torch.full((rows, o), 7.0, dtype=dtype, device="cuda"))
    new = lambda want_x: M.LayerGrad(torch.full((rows, i), 7.0, dtype=dtype, device="cuda") if want_x else None,
                                     torch.full((groups, o, i), 7.0, device="cuda"), torch.full((groups, o), 7.0, device="cuda"))
    both = M.layer_grouped_grad(x, w, gz, off, relu_input=True, out=new(True))
    plain = M.layer_grouped_grad(x, w, gz, off, want_x=False, out=new(False))
    for t in (y, both.x):
        assert (t[:3] == 7.0).all() and (t[ends[-1]:] == 7.0).all()
    for g, (a, z) in enumerate(zip(ends, ends[1:])):
        xg, zg, wd = x[a:z], gz[a:z], w[g].double().t().contiguous()
        for s in range(0, z - a, ROWS):
            xd = xg[s:s + ROWS].double()
            want, size = torch.mm(xd, wd) + b[g].double(), torch.mm(xd.abs(), wd.abs()) + b[g].double().abs()
            near(y[a:z][s:s + ROWS], want.clamp_min(0), sums(i) * size + ROUND[dtype] * want.abs(), f"y of group {g}, rows from {s}")
        check_input(both.x[a:z], zg, w[g], lambda s, e: xg[s:e] > 0, dtype, f"of group {g}")
        for got in (both, plain):
            check_weights(got.weight[g], got.bias[g], zg, lambda s, e: xg[s:e].double(), f"of group {g}")


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", PACKED)
def test_packed(n, i, o, dtype, rectified):
    print(f"layer_grad_packed n={n} {i}->{o} {dtype} rectified {rectified}", flush=True)
    x, w, _, gz = inputs(n, 1, i, o, dtype, n + i + o)
    p = M.pack_activations(x, rectified=rectified)
    step = lambda a, z: torch.exp2(p.exponents[a:z].double() - 127).repeat_interleave(32, 1)[:, :i]
    v = lambda a, z: p.codes[a:z].double() * step(a, z)
    both = M.layer_grad_packed(p, w[0], gz, relu_input=rectified)
    check_input(both.x, gz, w[0], (lambda a, z: p.codes[a:z] > 0) if rectified else None, dtype, "")
    for got in (both, M.layer_grad_packed(p, w[0], gz, want_x=False)):
        check_weights(got.weight, got.bias, gz, v, "")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", INT8)
def test_int8(n, i, o, dtype):
    """float32(sum) * x_scale and the product with weight_scale, a power of two here, are exact steps; so fma's rounding is a sum's."""
    print(f"layer_int8 n={n} {i}->{o} {dtype}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(n + i)
    code = lambda *s: torch.randint(-128, 128, s, generator=g, device="cuda").to(torch.int8)
    x, w = M.Quantized(code(n, i), torch.rand(n, generator=g, device="cuda") * 0.1), M.Quantized(code(o, i), torch.empty(o, device="cuda"))
    w.scale.copy_(torch.exp2(torch.randint(-9, -5, (o,), generator=g, device="cuda").float()))
    b = torch.randn(o, generator=g, device="cuda")
    got, wd = M.layer_int8(x, w, b, dtype=dtype), w.codes.double().t().contiguous()
    for a in range(0, n, ROWS):
        total = torch.mm(x.codes[a:a + ROWS].double(), wd).float()
        want = ((total * x.scale[a:a + ROWS, None]) * w.scale + b).clamp_min(0).to(dtype)
        assert torch.equal(got[a:a + ROWS], want), f"{int((got[a:a + ROWS] != want).sum())} differ, rows from {a}"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,i,o", GROUPED)
def test_grouped_poison(sizes, i, o, dtype):
    """Not finite: rows of no group, the workspace, and then one value of the largest group's x and one of its g_z. Nothing else changes."""
    n, groups = sum(sizes), len(sizes)
    print(f"grouped n={n} in {groups} {i}->{o} {dtype}", flush=True)
    ends = [9]
    for s in sizes:
        ends.append(ends[-1] + s)
    taken = slice(9, ends[-1])
    x, w, b, gz = inputs(ends[-1] + 70, groups, i, o, dtype, n)
    off = torch.tensor(ends, device="cuda")
    clean, grads = M.layer_grouped(x, w, b, off, relu=False), M.layer_grouped_grad(x, w, gz, off)
    for t in (x, gz):
        t[:9], t[ends[-1]:] = math.nan, math.nan
    need = _layers.load().maestro_layer_grouped_grad_workspace(len(x), groups, i, o, int(dtype == torch.bfloat16))
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    used = M.layer_grouped_grad(x, w, gz, off, workspace=ws[:need])
    assert (ws[need:] == 0xFF).all()
    assert torch.equal(M.layer_grouped(x, w, b, off, relu=False)[taken], clean[taken]) and torch.equal(used.x[taken], grads.x[taken])
    assert torch.equal(used.weight, grads.weight) and torch.equal(used.bias, grads.bias)
    g = max(range(groups), key=lambda k: sizes[k])
    bad = (ends[g] + ends[g + 1]) // 2
    x[bad, i - 1], gz[bad, o - 1] = math.nan, math.inf
    rest = torch.ones(len(x), dtype=torch.bool, device="cuda")
    rest[bad], rest[:9], rest[ends[-1]:] = False, False, False
    assert torch.equal(M.layer_grouped(x, w, b, off, relu=False)[rest], clean[rest])
    dirty = M.layer_grouped_grad(x, w, gz, off, workspace=ws[:need])
    assert torch.equal(dirty.x[rest], grads.x[rest])
    others = [k for k in range(groups) if k != g]
    assert torch.equal(dirty.weight[others], grads.weight[others]) and torch.equal(dirty.bias[others], grads.bias[others])
    assert torch.equal(dirty.weight[g, :-1, :-1], grads.weight[g, :-1, :-1]) and torch.equal(dirty.bias[g, :-1], grads.bias[g, :-1])
    assert torch.isnan(dirty.weight[g, :, -1]).all() and torch.isinf(dirty.bias[g, -1])


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", PACKED)
def test_packed_poison(n, i, o, dtype, rectified):
    """Not finite: the workspace, and then 32 values kept and one of g_z. They spoil their columns and their row of g_w, and their row of g_x."""
    print(f"layer_grad_packed n={n} {i}->{o} {dtype} rectified {rectified}", flush=True)
    x, w, _, gz = inputs(n, 1, i, o, dtype, n)
    p = M.pack_activations(x, rectified=rectified)
    need = _layers.load().maestro_layer_grad_packed_workspace(n, i, o, int(dtype == torch.bfloat16))
    clean = M.layer_grad_packed(p, w[0], gz, relu_input=rectified)
    p.codes[n // 3, :32], p.exponents[n // 3, 0] = 0, 255
    gz[n // 2, o - 1] = math.nan
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    dirty = M.layer_grad_packed(p, w[0], gz, relu_input=rectified, workspace=ws[:need])
    assert (ws[need:] == 0xFF).all()
    assert torch.equal(dirty.weight[:-1, 32:], clean.weight[:-1, 32:]) and torch.equal(dirty.bias[:-1], clean.bias[:-1])
    assert torch.isnan(dirty.weight[:, :32]).all() and torch.isnan(dirty.weight[-1]).all() and torch.isnan(dirty.bias[-1])
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[[n // 3, n // 2]] = False
    assert torch.equal(dirty.x[rest], clean.x[rest]) and torch.equal(dirty.x[n // 3, 32:], clean.x[n // 3, 32:])
