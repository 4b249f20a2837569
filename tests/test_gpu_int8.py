"""maestro_quantize_rows and maestro_layer_int8 against their definitions, bit for bit: codes from the real quotient (float64
decides it: two float32 a 2^-24 of their size apart have quotients further from a tie than 2^-30), whole-number sums in
int64, and the float32 steps in the documented order; the fused multiply-add in 64 bits of mantissa, where its product is exact."""
import math

import numpy as np
import pytest
import torch

import paper_2606_12950_amd as M

pytestmark = pytest.mark.gpu


def quantized(x):
    """The definition, on the CPU."""
    x = x.double()
    scale = (x.abs().amax(1) / 127).float().clamp_min(2.0 ** -126)
    q = torch.round(x / scale.double()[:, None])
    bad = ~torch.isfinite(x).all(1)
    scale[bad] = math.nan
    return torch.where(bad[:, None], 0.0, q).to(torch.int8), scale


def same(got, want):
    codes, scale = want
    assert torch.equal(got.codes.cpu(), codes), f"{int((got.codes.cpu() != codes).sum())} of {codes.numel()} codes"
    assert torch.equal(got.scale.cpu().view(torch.int32), scale.view(torch.int32)) or \
        torch.equal(torch.nan_to_num(got.scale.cpu(), nan=-1.0), torch.nan_to_num(scale, nan=-1.0))


SHAPES = [(1, 16), (3, 16), (2, 32), (5, 48), (7, 80), (63, 256), (65, 272), (129, 512), (300, 1024), (17, 1040), (33, 4096), (6, 4112),
          (3, 16384), (4099, 64), (20011, 128)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d", SHAPES)
def test_quantize_rows(n, d, dtype):
    print(f"quantize n={n} d={d} {dtype}", flush=True)
    g = torch.Generator().manual_seed(n + d)
    x = (torch.randn(n, d, generator=g) * torch.exp(3 * torch.randn(n, 1, generator=g))).to(dtype)
    same(M.quantize_rows(x.cuda()), quantized(x))


def test_rows_of_several_launches():
    """More rows than 32 bits count threads of, at 64 a row, and codes past 2^34 bytes: every row is written, from its own row."""
    n, d = (1 << 26) + 5, 272
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 64 GiB")
    rows = torch.tensor([0, 1, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, (1 << 26) - 1, 1 << 26, n - 1])
    g = torch.Generator().manual_seed(9)
    some = torch.randn(len(rows), d, generator=g).bfloat16()
    x = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    x[rows.cuda()] = some.cuda()
    out = M.Quantized(torch.full((n, d), 77, dtype=torch.int8, device="cuda"), torch.full((n,), -1.0, device="cuda"))
    M.quantize_rows(x, out=out)
    same(M.Quantized(out.codes[rows.cuda()], out.scale[rows.cuda()]), quantized(some))
    out.scale[rows.cuda()] = 2.0 ** -126
    assert (out.scale == 2.0 ** -126).all()
    out.codes[rows.cuda()] = 0
    for part in out.codes.split(1 << 24):
        assert not part.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_hard_rows(dtype):
    """Ties, zeros, the smallest and largest values, NaN and infinities."""
    d = 64
    rows = [torch.zeros(d), torch.full((d,), -0.0), torch.linspace(-127, 127, d), torch.full((d,), 1e-45), torch.full((d,), -3e-39)]
    ties = torch.cat([torch.arange(-31.5, 32.5, 1.0)])
    ties[0] = 127.0                                   # scale 1: every other value halfway between two codes
    rows += [ties, ties * 2.0 ** -120, ties * 2.0 ** 120]
    rows += [torch.tensor([127.0, 63.5, 0.5, -0.5, 1.5, 2.5, -2.5, 126.5] * 8) * s for s in (1.0, 3.0, 2.0 ** -130)]
    rows += [torch.full((d,), 3.3e38), torch.tensor([1.0, -1.0] * 32), torch.tensor([2.0 ** -126, 2.0 ** -149] * 32)]
    for bad in (math.nan, math.inf, -math.inf):
        r = torch.ones(d)
        r[5] = bad
        rows.append(r)
    both = torch.ones(d)
    both[0], both[63] = math.inf, math.nan
    x = torch.stack([*rows, both]).to(dtype)
    got = M.quantize_rows(x.cuda())
    same(got, quantized(x))
    assert torch.isnan(got.scale[-4:]).all() and not got.codes[-4:].any()


def test_quantize_near_ties():
    """Values one float32 step around (m + 1/2) scale, for scales of many mantissas."""
    g = torch.Generator().manual_seed(2)
    most = (torch.rand(512, 1, generator=g) + 1) * 2.0 ** torch.randint(-20, 20, (512, 1), generator=g)
    scale = (most.double() / 127).float()
    m = torch.randint(-126, 126, (512, 63), generator=g)
    x = ((m + 0.5).double() * scale.double()).float()
    x = torch.where(torch.rand(512, 63, generator=g) < 0.5, torch.nextafter(x, torch.tensor(math.inf)), x)
    x = torch.where(torch.rand(512, 63, generator=g) < 0.3, torch.nextafter(x, torch.tensor(-math.inf)), x)
    x = torch.cat([most, x], 1).contiguous()
    same(M.quantize_rows(x.cuda()), quantized(x))


def definition(x, w, bias, relu, dtype):
    """fma(sum * x_scale, weight_scale, bias) in float32, rounded to dtype."""
    assert np.finfo(np.longdouble).nmant >= 63
    total = (x.codes.double() @ w.codes.double().t()).float()        # whole numbers below 2^53, rounded once
    part = (total * x.scale[:, None]).numpy().astype(np.longdouble)
    y = torch.from_numpy((part * w.scale.numpy().astype(np.longdouble) + bias.numpy().astype(np.longdouble)).astype(np.float32))
    if relu:
        y = torch.where(y < 0, 0.0, y)
    return y.to(dtype)


def equal(got, want, what):
    got = got.cpu()
    fine = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert fine.all(), f"{what}: {int((~fine).sum())} of {fine.numel()} differ, first at {(~fine).nonzero()[0].tolist()}"


def draw(n, i, o, seed):
    g = torch.Generator().manual_seed(seed)
    code = lambda *s: torch.randint(-128, 128, s, generator=g).to(torch.int8)
    return (M.Quantized(code(n, i), torch.rand(n, generator=g) * 0.1), M.Quantized(code(o, i), torch.rand(o, generator=g) * 0.01),
            torch.randn(o, generator=g))


def on_gpu(q):
    return M.Quantized(q.codes.cuda(), q.scale.cuda())


SIZES = [(1, 16, 16), (2, 32, 16), (15, 16, 48), (17, 48, 80), (63, 64, 128), (65, 272, 16), (127, 16, 512), (128, 512, 512),
         (129, 144, 176), (257, 256, 272), (300, 256, 512), (511, 80, 1024), (1000, 1024, 64), (1, 1024, 1024), (4099, 512, 64),
         (20011, 256, 512), (9000, 1024, 1024), (70001, 64, 48), (140000, 64, 272), (8, 16384, 32), (5, 32, 16384)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,i,o", SIZES)
def test_layer_int8(n, i, o, dtype):
    print(f"layer_int8 n={n} {i}->{o} {dtype}", flush=True)
    x, w, b = draw(n, i, o, n + i + o)
    for relu in (False, True):
        got = M.layer_int8(on_gpu(x), on_gpu(w), b.cuda(), relu=relu, dtype=dtype)
        assert got.dtype == dtype
        equal(got, definition(x, w, b, relu, dtype), f"relu {relu}")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_rounds(dtype):
    """3,128 tiles of 256 x 256, rows of every workgroup's first, a middle and its last one."""
    n, i, o = 200000, 48, 1024
    x, w, b = draw(n, i, o, 5)
    got = M.layer_int8(on_gpu(x), on_gpu(w), b.cuda(), relu=False, dtype=dtype)
    for first in (0, 777, 99999, 131000, n - 600):
        rows = slice(first, first + 600)
        equal(got[rows], definition(M.Quantized(x.codes[rows], x.scale[rows]), w, b, False, dtype), f"rows from {first}")


def test_largest_sums():
    """16,384 products of -128 and -128: 2^28."""
    x = M.Quantized(torch.full((3, 16384), -128, dtype=torch.int8), torch.ones(3))
    w = M.Quantized(torch.full((16, 16384), -128, dtype=torch.int8), torch.ones(16))
    got = M.layer_int8(on_gpu(x), on_gpu(w), torch.zeros(16, device="cuda"), dtype=torch.float32)
    assert (got == 2.0 ** 28).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_bad_row_stays_one(dtype):
    """A row of NaN scale gives NaN throughout, also rectified, and no other row changes; nothing past the last is written."""
    x, w, b = draw(200, 64, 48, 3)
    clean = M.layer_int8(on_gpu(x), on_gpu(w), b.cuda(), dtype=dtype)
    x.scale[[0, 64, 199]] = math.nan
    buf = torch.full((208, 48), 7.0, dtype=dtype, device="cuda")
    dirty = M.layer_int8(on_gpu(x), on_gpu(w), b.cuda(), dtype=dtype, out=buf[:200])
    bad = torch.isnan(x.scale).cuda()
    assert torch.isnan(dirty[bad]).all() and torch.equal(clean[~bad], dirty[~bad]) and (buf[200:] == 7.0).all()


def test_no_rows():
    q = M.quantize_rows(torch.empty(0, 64, device="cuda"))
    assert q.codes.shape == (0, 64) and q.scale.shape == (0,)
    _, w, b = draw(1, 64, 32, 1)
    assert M.layer_int8(q, on_gpu(w), b.cuda()).shape == (0, 32)


def test_near_the_layer():
    """A layer of the values that the codes stand for: the difference to the float layer is the quantisation's, for each
    product at most |x| s_w / 2 + |w| s_x / 2 + s_x s_w / 4, and the rounding of the outputs."""
    g = torch.Generator().manual_seed(4)
    x, w, b = torch.randn(300, 256, generator=g), torch.randn(64, 256, generator=g) / 16, torch.randn(64, generator=g)
    xq, wq = M.quantize_rows(x.cuda()), M.quantize_rows(w.cuda())
    got = M.layer_int8(xq, wq, b.cuda(), relu=False, dtype=torch.float32).cpu().double()
    sx, sw = xq.scale.cpu().double()[:, None], wq.scale.cpu().double()
    tol = x.double().abs().sum(1, keepdim=True) * sw / 2 + w.double().abs().sum(1) * sx / 2 + 256 * sx * sw / 4 + 2.0 ** -20
    assert ((got - (x.double() @ w.double().t() + b.double())).abs() <= tol).all()
