"""maestro_layer and maestro_layer_grad in bfloat16 at sizes that take the largest tiles: workgroups that make several tiles,
of one to many stages of k, with ragged edges, against float64 on the GPU in blocks of rows; and float32 with more tiles than
workgroups. Bounds as in test_gpu_layers."""
import math

import pytest
import torch

import paper_2606_12950_amd as M

pytestmark = pytest.mark.gpu
ROWS = 1 << 14

# 256 x 256 tiles for the activations need d_out > 128 and 512 of them, for the input's gradient d_in > 128 and 512, for the
# weights' gradient both > 128 and 131,072 rows. Stages of 64 k (32 for the weights' gradient).
FORWARD = [(70_001, 48, 272), (131_073, 64, 256), (70_003, 80, 272), (66_000, 128, 400), (65_541, 192, 272), (65_601, 528, 1040)]
INPUT = [(66_001, 272, 48), (131_073, 256, 64), (66_000, 400, 80), (65_541, 272, 128), (65_601, 1040, 528)]
WEIGHT = [(131_101, 272, 272), (131_073, 144, 656), (140_000, 528, 144), (262_139, 256, 256),
          (131_089, 2064, 2064)]                                  # more values to join than one round of workgroups takes


def inputs(n, i, o, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return r(n, i).bfloat16(), (r(o, i) * i ** -0.5).bfloat16(), r(o), (r(n, o) / n).bfloat16()


def near(got, want, tol, what):
    off = (got.double() - want).abs()
    wrong = ~(off <= tol)
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} off, first at {wrong.nonzero()[0].tolist()}"


def sums(k):
    return 2.0 ** -24 * (32 + 2 * math.sqrt(k))


@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("n,i,o", FORWARD)
def test_layer(n, i, o, relu):
    print(f"layer n={n} {i}->{o} relu={relu}", flush=True)
    x, w, b, _ = inputs(n, i, o, n + i)
    y, again = M.layer(x, w, b, relu=relu), M.layer(x, w, b, relu=relu)
    assert torch.equal(y, again)
    wd = w.double().t().contiguous()
    for a in range(0, n, ROWS):
        xd = x[a:a + ROWS].double()
        z = torch.mm(xd, wd) + b.double()
        tol = sums(i) * (torch.mm(xd.abs(), wd.abs()) + b.double().abs()) + 2.0 ** -8 * z.abs()
        near(y[a:a + ROWS], z.clamp_min(0) if relu else z, tol, f"rows from {a}")


@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("n,i,o", INPUT)
def test_input_gradient(n, i, o, relu):
    print(f"layer_grad n={n} {i}->{o} relu_input={relu}", flush=True)
    x, w, _, gz = inputs(n, i, o, n + o)
    gx, again = (M.layer_grad(x, w, gz, relu_input=relu).x for _ in range(2))
    assert torch.equal(gx, again)
    wd = w.double()
    for a in range(0, n, ROWS):
        gd = gz[a:a + ROWS].double()
        want = torch.mm(gd, wd)
        tol = sums(o) * torch.mm(gd.abs(), wd.abs()) + 2.0 ** -8 * want.abs()
        if relu:
            want = torch.where(x[a:a + ROWS] > 0, want, 0.0)
        near(gx[a:a + ROWS], want, tol, f"rows from {a}")


@pytest.mark.parametrize("n,i,o", WEIGHT)
def test_weights_gradient(n, i, o):
    print(f"layer_grad n={n} {i}->{o} weights", flush=True)
    x, w, _, gz = inputs(n, i, o, n + i + o)
    one, two = (M.layer_grad(x, w, gz, want_x=False) for _ in range(2))
    assert torch.equal(one.weight, two.weight) and torch.equal(one.bias, two.bias)
    gw = torch.zeros(o, i, dtype=torch.float64, device="cuda")
    size, gb, gb_size = torch.zeros_like(gw), torch.zeros(o, dtype=torch.float64, device="cuda"), torch.zeros(o, dtype=torch.float64, device="cuda")
    for a in range(0, n, ROWS):
        xd, gd = x[a:a + ROWS].double(), gz[a:a + ROWS].double()
        gt = gd.t().contiguous()
        gw += torch.mm(gt, xd)
        size += torch.mm(gt.abs(), xd.abs())
        gb += gd.sum(0)
        gb_size += gd.abs().sum(0)
    near(one.weight, gw, sums(n) * size, "weight")
    near(one.bias, gb, sums(n) * gb_size, "bias")


@pytest.mark.parametrize("relu", [False, True])
def test_float32_tiles_in_a_second_round(relu):
    """More tiles than the 65,536 workgroups of a launch."""
    n, i, o = 64 * 65_536 + 67, 16, 32
    print(f"layer n={n} {i}->{o} float32 relu={relu}", flush=True)
    x, w, b, gz = (t.float() for t in inputs(n, i, o, 7))
    y, gx = M.layer(x, w, b, relu=relu), M.layer_grad(x, w, gz, relu_input=relu).x
    wd = w.double()
    wt = wd.t().contiguous()
    for a in range(0, n, 1 << 20):
        xd, gd = x[a:a + (1 << 20)].double(), gz[a:a + (1 << 20)].double()
        z, back = torch.mm(xd, wt) + b.double(), torch.mm(gd, wd)
        near(y[a:a + (1 << 20)], z.clamp_min(0) if relu else z,
             sums(i) * (torch.mm(xd.abs(), wt.abs()) + b.double().abs()) + 2.0 ** -23 * z.abs(), f"y from row {a}")
        near(gx[a:a + (1 << 20)], torch.where(xd > 0, back, 0.0) if relu else back,
             sums(o) * torch.mm(gd.abs(), wd.abs()) + 2.0 ** -23 * back.abs(), f"g_x from row {a}")
