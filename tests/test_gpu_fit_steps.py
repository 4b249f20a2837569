"""What Fit.step gives back and leaves behind: every step's own norm."""
import pytest
import torch

from paper_2606_12950_amd import fit as F
from test_gpu_fit import network

pytestmark = pytest.mark.gpu
NETWORKS = [((64, 128, 32), torch.float32), ((256, 512, 64), torch.bfloat16)]


def batch(dims, dtype, n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, dims[0], generator=g).to(dtype).cuda()
    return x, torch.randint(-1, dims[-1], (n,), generator=g, dtype=torch.int32).cuda()


def test_every_step_has_its_own_norm():
    dims, dtype = NETWORKS[0]
    f = F.Fit(*network(dims, dtype, 1), 100)
    kept, seen = [], []
    for s in range(4):
        mean, norm = f.step(*batch(dims, dtype, 100, s), 0.1)
        kept.append((mean, norm))
        seen.append((mean.item(), norm.item()))
    assert [(m.item(), n.item()) for m, n in kept] == seen and len(set(seen)) == 4
