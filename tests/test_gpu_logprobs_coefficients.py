"""maestro_logprobs_grad with entropy coefficients up to float32's largest, against float64 with test_gpu_logprobs's bounds."""
import pytest
import torch

import paper_2606_12950_amd as M
from test_gpu_logprobs import INF, grad_bound, grad_reference, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [40, 300, 3000, 20000])
def test_largest_coefficients(v, dtype):
    """Masked logits get 0, and unlikely ones a product that is in range though coefficient times ln p is not. p stays
    above float32's least normal number (x within 85 of the maximum, ln S < 2.5)."""
    n = 24
    g = torch.Generator().manual_seed(v)
    x = -85.0 * torch.rand(n, v, generator=g) ** 0.3
    x[:, 0] = 0.0
    x[torch.rand(n, v, generator=g) < 0.3] = -INF
    x[:, 1] = 0.0
    x[::5, 2:] = -INF
    x = x.to(dtype)
    token = torch.randint(-1, v, (n,), generator=g, dtype=torch.int32)
    ge = torch.full((n,), 3e38) * torch.tensor([1.0, -1.0]).repeat(n // 2)
    gl = torch.randn(n, generator=g)
    _, h, _, _, m, ls = reference(x, token, 0)
    assert ls.max() < 2.5
    dev = torch.stack([m, ls], 1).float().cuda(), h.float().cuda()
    for t, a in ((token, gl), (None, None)):
        got = M.logprobs_grad(x.cuda(), None if t is None else t.cuda(), *dev, None if a is None else a.cuda(), ge.cuda()).cpu()
        assert (got[(x == -INF) & (torch.arange(v) != token[:, None])] == 0).all()
        want, bound = grad_reference(x, token, a, ge)[0], grad_bound(x, token, a, ge)
        want = torch.where(want.abs() > torch.finfo(dtype).max, want.sign() * INF, want)
        wrong = ~((got.double() == want) | ((got.double() - want).abs() <= bound))
        assert not wrong.any(), (int(wrong.sum()), wrong.nonzero()[0].tolist(), got[wrong][0].item(), want[wrong][0].item())
