"""maestro_logprobs and maestro_logprobs_grad where a workgroup takes more than one row, or part of one, after the other: sizes
just past what one round of each form's workgroups takes, against the definition in float64 on the GPU.

Bounds as in test_gpu_logprobs (there the sums are chains of at most 512 additions and a tree: 640 with the logarithm).
In general a chain is of v / 64 additions where a wavefront takes a row and of v / 256 where 256 threads do, so
2^-24 (4 |l| + max(640, chain + 128))."""
import math

import pytest
import torch

import paper_2606_12950_amd as M
from test_gpu_logprobs import INF, U, grad_bound, grad_reference, reference

pytestmark = pytest.mark.gpu


def draw(n, v, dtype, seed, masked=0.2):
    """On the GPU: logits of spread 2.5 in few steps (ties), one row in 61 masked throughout, one in 127 spoilt."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(n, v, generator=g, device="cuda") * 2.5
    if masked:
        x.masked_fill_(torch.rand(n, v, generator=g, device="cuda") < masked, -INF)
    x = x.to(dtype)
    x[::61] = -INF
    x[::127, v // 2] = math.nan
    return x, torch.randint(-1, v + 1, (n,), generator=g, dtype=torch.int32, device="cuda")


def close(got, want, bound, what):
    got = got.double()
    wrong = ~((got == want) | (torch.isnan(got) & torch.isnan(want)) | ((got - want).abs() <= bound))
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} off, first at {wrong.nonzero()[0].tolist()}: " \
        f"{got[wrong][0].item()} for {want[wrong][0].item()}"


def check(n, v, k, dtype, chain, masked=0.2):
    x, token = draw(n, v, dtype, n + v, masked)
    got = M.logprobs(x, token, k=k)
    sums = max(640, chain + 128)
    rows = max(1, (1 << 24) // v)
    for a in range(0, n, rows):
        b = min(n, a + rows)
        lp, h, ids, top, m, ls = reference(x[a:b], token[a:b], k)
        close(got.logprob[a:b], lp, U * (4 * lp.abs() + sums), f"logprob from row {a}")
        close(got.entropy[a:b], h, U * (sums + 16 * h) * (1 + h), f"entropy from row {a}")
        assert torch.equal(got.top_id[a:b], ids), f"ids from row {a}"
        close(got.top_logprob[a:b], top, U * (4 * top.abs() + sums), f"top_logprob from row {a}")
        close(got.stats[a:b, 0], m, 0.0, f"max from row {a}")
        close(got.stats[a:b, 1], ls, U * (4 * ls.abs() + sums), f"ln S from row {a}")


@pytest.mark.parametrize("n,v,k,dtype", [
    (262_147, 13, 4, torch.float32), (262_147, 64, 4, torch.bfloat16), (131_075, 100, 3, torch.bfloat16),
    (65_539, 100, 5, torch.float32), (32_771, 500, 5, torch.bfloat16), (16_387, 1000, 4, torch.bfloat16),
    (8_197, 1100, 2, torch.bfloat16), (8_197, 700, 2, torch.float32)])
def test_rows_in_registers(n, v, k, dtype):
    print(f"logprobs rows after rows n={n} v={v} k={k} {dtype}", flush=True)
    check(n, v, k, dtype, 0)


@pytest.mark.parametrize("n,v,k,dtype", [
    (8_195, 4096, 6, torch.bfloat16), (16_390, 2048, 16, torch.float32), (8_200, 9000, 5, torch.bfloat16),      # a wavefront
    (2_051, 10_300, 6, torch.float32), (2_050, 40_001, 16, torch.bfloat16)])                                   # 256 threads
def test_rows_of_a_workgroup(n, v, k, dtype):
    print(f"logprobs jobs after jobs n={n} v={v} k={k} {dtype}", flush=True)
    check(n, v, k, dtype, v // 64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_sums(dtype):
    """Rows that 256 threads take in chains of more than 512 additions."""
    n, v = 257, 300_001
    print(f"logprobs long sums n={n} v={v} {dtype}", flush=True)
    check(n, v, 4, dtype, v // 256, masked=0.0)


@pytest.mark.parametrize("n,v,dtype", [(65_541, 520, torch.bfloat16),                      # a wavefront to a row
                                       (8_200, 8200, torch.bfloat16), (16_390, 2060, torch.float32),      # parts of rows
                                       (524_291, 64, torch.bfloat16)])                     # rows end to end
@pytest.mark.parametrize("entropy", [True, False])
def test_gradient(n, v, dtype, entropy):
    print(f"logprobs_grad rows after rows n={n} v={v} {dtype}", flush=True)
    x, token = draw(n, v, dtype, n + v)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    gl = torch.randn(n, generator=g, device="cuda")
    ge = torch.randn(n, generator=g, device="cuda") if entropy else None
    rows = max(1, (1 << 23) // v)
    parts = [reference(x[a:a + rows], token[a:a + rows], 0) for a in range(0, n, rows)]
    h, m, ls = (torch.cat([p[i] for p in parts]) for i in (1, 4, 5))
    got = M.logprobs_grad(x, token, torch.stack([m, ls], 1).float(), h.float(), gl, ge)
    for a in range(0, n, rows):
        own = slice(a, min(n, a + rows))
        want, bound = expected(x[own], token[own], gl[own], None if ge is None else ge[own])
        close(got[own], want, bound, f"grad from row {a}")


def expected(x, token, g, ge):
    with torch.device("cuda"):                # the reference's own new tensors too
        return grad_reference(x, token, g, ge)[0], grad_bound(x, token, g, ge)
