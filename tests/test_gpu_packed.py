"""maestro_pack_activations, maestro_unpack_activations and maestro_layer_grad_packed.

Codes, exponents and values are compared bit for bit with the definition in float64 on the CPU (quotients by powers of two are
exact there). The gradients are those of maestro_layer_grad for the values held, which the type holds exactly; bounds as there:
2^-24 (32 + 2 sqrt(K)) sum |a b| for a sum of K products, and one rounding of g_x."""
import math

import pytest
import torch

import paper_2606_12950_amd as M

pytestmark = pytest.mark.gpu
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def packed(x, rectified):
    """The definition: for every 32 values of a row the least exponent from 1 on whose codes are in range."""
    n, d = x.shape
    most = 255 if rectified else 127
    v = torch.nn.functional.pad(x.double(), (0, -d % 32)).view(n, -1, 32)
    if rectified:
        v = torch.where(v <= 0, 0.0, v)
    bad = ~torch.isfinite(v).all(2)
    v = torch.where(bad[:, :, None], 0.0, v)
    big = v.abs().amax(2)
    e = torch.ones_like(big)
    for k in range(1, 255):
        e = torch.where((e == k) & (torch.round(big * 2.0 ** (127 - k)) > most), k + 1.0, e)
    q = torch.round(v * torch.exp2(127 - e)[:, :, None])
    if rectified:
        q = torch.where((v > 0) & (q < 1), 1.0, q)
    e = torch.where(bad, 255.0, e)
    return q.view(n, -1)[:, :d].to(torch.uint8 if rectified else torch.int8), e.to(torch.uint8)


def values(codes, exponents):
    s = torch.where(exponents == 255, math.inf, torch.exp2(exponents.double() - 127)).repeat_interleave(32, 1)[:, :codes.shape[1]]
    return codes.double() * s


def same_values(got, want):
    got = got.cpu().double()
    assert ((got == want) | (torch.isnan(got) & torch.isnan(want))).all()


def check(x, rectified):
    p = M.pack_activations(x.cuda(), rectified=rectified)
    codes, exponents = packed(x, rectified)
    assert p.codes.dtype == (torch.uint8 if rectified else torch.int8)
    assert torch.equal(p.exponents.cpu(), exponents), (p.exponents.cpu() != exponents).nonzero()[:4].tolist()
    assert torch.equal(p.codes.cpu(), codes), (p.codes.cpu() != codes).nonzero()[:4].tolist()
    for dtype in (torch.float32, torch.bfloat16):
        same_values(M.unpack_activations(p, dtype=dtype), values(codes, exponents))
    return p


SHAPES = [(1, 16), (3, 16), (2, 32), (5, 48), (7, 80), (63, 256), (65, 272), (129, 512), (300, 1024), (17, 1040), (3, 16384), (4099, 64),
          (20011, 112)]


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d", SHAPES)
def test_pack(n, d, dtype, rectified):
    print(f"pack n={n} d={d} {dtype} rectified {rectified}", flush=True)
    g = torch.Generator().manual_seed(n + d)
    x = (torch.randn(n, d, generator=g) * torch.exp(4 * torch.randn(n, 1, generator=g))).to(dtype)
    p = check(x, rectified)
    held = M.unpack_activations(p, dtype=torch.float32).cpu().double()
    want = x.double().clamp_min(0) if rectified else x.double()
    step = torch.exp2(p.exponents.cpu().double() - 127).repeat_interleave(32, 1)[:, :d]
    assert ((held - want).abs() <= (step if rectified else step / 2)).all()
    if rectified:
        assert torch.equal(p.codes.cpu() > 0, x > 0)


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pack_hard_blocks(dtype, rectified):
    """Largest values just below and at the next exponent, ties, zeros, the smallest and largest values, one value alone."""
    rows = [torch.zeros(32), torch.full((32,), -0.0)]
    for big in (127.0, 127.25, 127.49999, 127.5, 127.75, 128.0, 255.0, 255.49998, 255.5, 255.75, 256.0, 1.0):
        for s in (1.0, 2.0 ** -125, 2.0 ** 119, 2.0 ** -133, 2.0 ** -10):
            r = torch.arange(32) * 0.5 - 7.25
            r[3] = big
            rows.append(r * s)
    rows += [torch.full((32,), v) for v in (1e-45, -1e-45, 3.3e38, -3.3e38, 2.0 ** -127, 2.0 ** -126)]
    for at in (0, 15, 16, 31):
        r = torch.zeros(32)
        r[at] = 1e-3
        rows.append(r)
    check(torch.stack(rows).to(dtype), rectified)
    # as the two blocks of a row of 48: the last has 16 values
    x = torch.stack(rows)
    check(torch.cat([x[:-1], x[1:, :16]], 1).to(dtype).contiguous(), rectified)


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pack_not_finite(dtype, rectified):
    """A NaN or an infinity spoils its 32 values and no others."""
    x = torch.randn(6, 96, generator=torch.Generator().manual_seed(1)).to(dtype)
    x[0, 5], x[1, 40], x[2, 95], x[3, 31] = math.nan, math.inf, -math.inf, math.nan
    x[4, 0], x[4, 32] = math.inf, math.nan
    p = check(x, rectified)
    v = M.unpack_activations(p, dtype=dtype).cpu()
    spoilt = torch.isnan(v).view(6, 3, 32).all(2)
    want = torch.tensor([[1, 0, 0], [0, 1, 0], [0, 0, not rectified], [1, 0, 0], [1, 1, 0], [0, 0, 0]], dtype=torch.bool)
    assert torch.equal(spoilt, want) and torch.equal(torch.isnan(v).view(6, 3, 32).any(2), want)


def test_nothing_beside_and_empty():
    x = torch.randn(30, 80, device="cuda")
    codes, exponents = torch.full((32, 80), 9, dtype=torch.int8, device="cuda"), torch.full((32, 3), 9, dtype=torch.uint8, device="cuda")
    p = M.pack_activations(x, out=M.Packed(codes[:30], exponents[:30]))
    assert (codes[30:] == 9).all() and (exponents[30:] == 9).all()
    out = torch.full((32, 80), 7.0, device="cuda")
    M.unpack_activations(p, dtype=torch.float32, out=out[:30])
    assert (out[30:] == 7.0).all()
    e = M.pack_activations(torch.empty(0, 80, device="cuda"))
    assert e.codes.shape == (0, 80) and e.exponents.shape == (0, 3) and M.unpack_activations(e).shape == (0, 80)


def bound(a, b):
    """of the product a b, both float64"""
    return 2.0 ** -24 * (32 + 2 * math.sqrt(a.shape[1])) * (a.abs() @ b.abs())


def near(got, want, tol, what):
    off = (got.cpu().double() - want).abs()
    wrong = ~(off <= tol)
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} off, first at {wrong.nonzero()[0].tolist()}, " \
        f"by up to {(off / tol.clamp_min(1e-300))[wrong].max():.3g} of the bound"


def draw(n, i, o, dtype, rectified, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, i, generator=g) * torch.exp(torch.randn(n, 1, generator=g))
    codes, exponents = packed(x, rectified)
    return (codes, exponents, values(codes, exponents), (torch.randn(o, i, generator=g) * i ** -0.5).to(dtype),
            (torch.randn(n, o, generator=g) / max(n, 1)).to(dtype))


SIZES = [(1, 16, 16), (2, 32, 16), (15, 16, 48), (16, 64, 32), (17, 48, 80), (63, 64, 128), (65, 272, 16), (127, 16, 512), (128, 512, 512),
         (129, 144, 176), (257, 256, 272), (300, 256, 512), (511, 80, 1024), (1000, 1024, 64), (1, 1024, 1024), (31, 2048, 1040),
         (4096, 64, 128), (4099, 512, 64), (9000, 1024, 1024), (70001, 64, 48), (8, 16384, 32), (5, 32, 16384), (140003, 256, 272)]


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", SIZES)
def test_layer_grad_packed(n, i, o, dtype, rectified):
    print(f"layer_grad_packed n={n} {i}->{o} {dtype} rectified {rectified}", flush=True)
    codes, exponents, v, w, gz = draw(n, i, o, dtype, rectified, n + i + o)
    p = M.Packed(codes.cuda(), exponents.cuda())
    wd, gd = w.double(), gz.double()
    gx, gw, gb = gd @ wd, gd.t() @ v, gd.sum(0)
    for relu, want_x in ((False, True), (rectified, True), (rectified, False)):
        got = M.layer_grad_packed(p, w.cuda(), gz.cuda(), relu_input=relu, want_x=want_x)
        near(got.weight, gw, bound(gd.t(), v) + 1e-38, "weight")
        near(got.bias, gb, bound(gd.t(), torch.ones(n, 1, dtype=torch.float64))[:, 0] + 1e-38, "bias")
        assert (got.x is not None) == want_x
        if want_x:
            want = torch.where(v > 0, gx, 0.0) if relu else gx
            near(got.x, want, bound(gd, wd) + ROUND[dtype] * want.abs(), "x")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_grad_equal_calls_nothing_beside_and_empty(dtype):
    n, i, o = 700, 80, 96
    codes, exponents, _, w, gz = (t.cuda() for t in draw(n, i, o, dtype, True, 3))
    p = M.Packed(codes, exponents)
    first = M.layer_grad_packed(p, w, gz, relu_input=True)
    bx = torch.full((n + 8, i), 7.0, dtype=dtype, device="cuda")
    bw, bb = torch.full((o + 8, i), 7.0, device="cuda"), torch.full((o + 8,), 7.0, device="cuda")
    again = M.layer_grad_packed(p, w, gz, relu_input=True, out=M.LayerGrad(bx[:n], bw[:o], bb[:o]))
    assert all(torch.equal(a, z) for a, z in zip(first, again))
    assert (bx[n:] == 7.0).all() and (bw[o:] == 7.0).all() and (bb[o:] == 7.0).all()
    none = M.layer_grad_packed(M.Packed(codes[:0], exponents[:0]), w, gz[:0], relu_input=True)
    assert none.x.shape == (0, i) and not none.weight.any() and not none.bias.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_grad_of_values_not_finite(dtype):
    """NaN values spoil their columns of the weights' gradient and nothing else; their g_x is that of a zero."""
    n, i, o = 200, 96, 48
    codes, exponents, _, w, gz = draw(n, i, o, dtype, True, 5)
    clean = M.layer_grad_packed(M.Packed(codes.cuda(), exponents.cuda()), w.cuda(), gz.cuda(), relu_input=True)
    codes[130, 32:64], exponents[130, 1] = 0, 255
    dirty = M.layer_grad_packed(M.Packed(codes.cuda(), exponents.cuda()), w.cuda(), gz.cuda(), relu_input=True)
    assert torch.isnan(dirty.weight[:, 32:64]).all() and torch.equal(clean.bias, dirty.bias)
    rest = [c for c in range(i) if not 32 <= c < 64]
    assert torch.equal(clean.weight[:, rest], dirty.weight[:, rest])
    assert not dirty.x[130, 32:64].any() and torch.equal(clean.x[:130], dirty.x[:130]) and torch.equal(clean.x[131:], dirty.x[131:])


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,o", [(77, 48), (700, 96), (20011, 272)])
def test_grad_of_largest_and_smallest_steps(n, o, dtype, rectified):
    """A step for every 32 columns, from the smallest to the largest that packing gives; codes that fill them."""
    steps = torch.tensor([1, 2, 60, 127, 200, 240, *(e - rectified for e in (246, 247, 248, 249))], dtype=torch.uint8)
    i = 32 * len(steps)
    g = torch.Generator().manual_seed(n)
    codes = torch.randint(0, 256, (n, i), generator=g) if rectified else torch.randint(-127, 128, (n, i), generator=g)
    codes[:, -32:] = torch.div(codes[:, -32:], 2, rounding_mode="trunc")      # below 2^128
    codes = codes.to(torch.uint8 if rectified else torch.int8)
    exponents = steps.expand(n, -1).contiguous()
    v = values(codes, exponents)
    assert torch.isfinite(v.float()).all()
    w = (torch.randn(o, i, generator=g) * i ** -0.5).to(dtype)
    gz = (torch.randn(n, o, generator=g) * 2.0 ** -40).to(dtype)
    gd = gz.double()
    got = M.layer_grad_packed(M.Packed(codes.cuda(), exponents.cuda()), w.cuda(), gz.cuda())
    near(got.weight, gd.t() @ v, bound(gd.t(), v) + n * 2.0 ** -126, "weight")      # products below 2^-126 may count as 0


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_grad_of_infinite_steps(dtype, rectified):
    """Of codes that packing never gives, 1 and more of an infinite step: infinities, in their columns only."""
    n, i, o = 200, 96, 48
    codes, exponents, _, w, gz = draw(n, i, o, dtype, rectified, 7)
    clean = M.layer_grad_packed(M.Packed(codes.cuda(), exponents.cuda()), w.cuda(), gz.cuda())
    codes[130, 32:64], exponents[130, 1] = 5, 255
    assert (gz[130] != 0).all()
    dirty = M.layer_grad_packed(M.Packed(codes.cuda(), exponents.cuda()), w.cuda(), gz.cuda())
    assert torch.equal(dirty.weight[:, 32:64].cpu(), (gz[130].float() * math.inf)[:, None].expand(-1, 32))
    rest = [c for c in range(i) if not 32 <= c < 64]
    assert torch.equal(clean.weight[:, rest], dirty.weight[:, rest]) and torch.equal(clean.x, dirty.x)


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", [(300, 80, 48), (2001, 272, 80), (33001, 144, 272), (140003, 528, 272)])
def test_poison_in_large_layers(n, i, o, dtype, rectified):
    """32 values that are not finite and a gradient that is not spoil their columns, their row of g_w and their rows of g_x only."""
    g = torch.Generator().manual_seed(n)
    p = M.pack_activations(torch.randn(n, i, generator=g).to(dtype).cuda(), rectified=rectified)
    w, gz = (torch.randn(o, i, generator=g) * i ** -0.5).to(dtype).cuda(), (torch.randn(n, o, generator=g) / n).to(dtype).cuda()
    clean = M.layer_grad_packed(p, w, gz, relu_input=rectified)
    last = i - i % 32 or i - 32                                # the last exponent's columns
    p.codes[n - 1, last:], p.exponents[n - 1, -1] = 0, 255
    p.codes[64, :32], p.exponents[64, 0] = 0, 255
    gz[n // 2, o - 1] = math.nan
    ws = torch.full((1 << 28,), 0xFF, dtype=torch.uint8, device="cuda")
    dirty = M.layer_grad_packed(p, w, gz, relu_input=rectified, workspace=ws)
    assert torch.equal(dirty.weight[:-1, 32:last], clean.weight[:-1, 32:last]) and torch.equal(dirty.bias[:-1], clean.bias[:-1])
    assert torch.isnan(dirty.weight[:, :32]).all() and torch.isnan(dirty.weight[:, last:]).all() and torch.isnan(dirty.weight[-1]).all()
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[[64, n // 2, n - 1]] = False
    assert torch.isnan(dirty.bias[-1]) and torch.equal(dirty.x[rest], clean.x[rest])
    assert torch.equal(dirty.x[64, 32:], clean.x[64, 32:]) and torch.equal(dirty.x[n - 1, :last], clean.x[n - 1, :last])


@pytest.mark.parametrize("rectified", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d", [(7, 16), (40, 80), (2000, 112)])
def test_pack_of_the_largest_finite_values(n, d, dtype, rectified):
    """Finite values stay finite and within a step, up to the type's largest: where the least step that fits the codes would make
    2^128 of one, it is the step below, and codes past the last one are the last one."""
    most, top = 255 if rectified else 127, torch.finfo(dtype).max
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, d, generator=g) * 2.0 ** (120 + 7 * torch.rand(n, d, generator=g))
    limit = (most + 0.5) * 2.0 ** (120 if rectified else 121)                # from here on the definition's code is 2^128
    hard = torch.tensor([top, -top, limit, -limit, float(torch.nextafter(torch.tensor(limit), torch.tensor(0.0))), 1.0])
    x[torch.arange(n), torch.arange(n) % d] = hard[torch.arange(n) % 6]      # alone in its block, or beside others of its size
    x[n // 2] = top
    x = x.to(dtype)
    x = torch.where(torch.isinf(x), torch.tensor(top, dtype=dtype).copysign(x), x)
    assert torch.isfinite(x).all() and (x == top).any()
    p = M.pack_activations(x.cuda(), rectified=rectified)
    codes, exponents = p.codes.cpu().double(), p.exponents.cpu()
    v = x.double().clamp_min(0.0) if rectified else x.double()
    big = torch.nn.functional.pad(v, (0, -d % 32)).view(n, -1, 32).abs().amax(2)
    e = packed(x, rectified)[1].double()
    e = torch.where(big >= limit, e - 1, e)
    assert torch.equal(exponents.double(), e), (exponents.double() != e).nonzero()[:4].tolist()
    steps = torch.exp2(e - 127).repeat_interleave(32, 1)[:, :d]
    q = torch.round(v / steps).clamp(-most, most)
    if rectified:
        q = torch.where((v > 0) & (q < 1), 1.0, q)
    assert torch.equal(codes, q), (codes != q).nonzero()[:4].tolist()
    for to in (torch.float32, torch.bfloat16):
        held = M.unpack_activations(p, dtype=to).cpu()
        assert torch.isfinite(held).all() and torch.equal(held.double(), codes * steps)
        assert ((held.double() - v).abs() <= steps).all()
    # and the gradients of such values: w's are the sums of the values held
    o = 48
    gz = (torch.randn(n, o, generator=g) * 2.0 ** -30).to(dtype)
    w = torch.randn(o, d, generator=g).to(dtype)
    got = M.layer_grad_packed(p, w.cuda(), gz.cuda(), relu_input=rectified)
    gd, held = gz.double(), codes * steps
    near(got.weight, gd.t() @ held, bound(gd.t(), held) + n * 2.0 ** -126, "weight")
    want = torch.where(held > 0, gd @ w.double(), 0.0) if rectified else gd @ w.double()
    near(got.x, want, bound(gd, w.double()) + ROUND[dtype] * want.abs(), "x")
