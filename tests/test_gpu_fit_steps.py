"""What Fit.step gives back and leaves behind: every step's own norm, weights that a batch without finite gradients does not
touch, and stages without an observed length that take no part whatever their features hold."""
import math

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


def state(f):
    return [t.clone() for t in (*f.weights, *f.biases, *f.masters, *f.velocity)]


def test_every_step_has_its_own_norm():
    dims, dtype = NETWORKS[0]
    f = F.Fit(*network(dims, dtype, 1), 100)
    kept, seen = [], []
    for s in range(4):
        mean, norm = f.step(*batch(dims, dtype, 100, s), 0.1)
        kept.append((mean, norm))
        seen.append((mean.item(), norm.item()))
    assert [(m.item(), n.item()) for m, n in kept] == seen and len(set(seen)) == 4


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dims,dtype", NETWORKS)
def test_a_step_without_finite_gradients_changes_nothing(dims, dtype, bad):
    n, fits = 100, []
    for with_bad in (False, True):
        f = F.Fit(*network(dims, dtype, 2), n)
        f.step(*batch(dims, dtype, n, 1), 0.1)
        if with_bad:
            before = state(f)
            x, bins = batch(dims, dtype, n, 2)
            x[5], bins[5] = bad, 3
            mean, norm = f.step(x, bins, 0.1)
            assert not math.isfinite(mean.item()) and not math.isfinite(norm.item())
            assert all(map(torch.equal, state(f), before))
        f.step(*batch(dims, dtype, n, 3), 0.1)
        fits.append(state(f))
    assert all(map(torch.equal, *fits)) and all(t.isfinite().all() for t in fits[0])


@pytest.mark.parametrize("dims,dtype", NETWORKS)
def test_unobserved_stages_take_no_part(dims, dtype):
    n, got = 200, []
    for features in (0.0, 1.0, math.nan, math.inf):
        f = F.Fit(*network(dims, dtype, 3), n)
        x, bins = batch(dims, dtype, n, 4)
        bins[17], bins[150] = -1, dims[-1]
        x[17], x[150, 3] = features, features
        x[150, :3] = 0.0
        mean, norm = f.step(x, bins, 0.1)
        got.append([mean, norm, *state(f)])
    for other in got[1:]:
        assert all(map(torch.equal, other, got[0]))
    assert all(t.isfinite().all() for t in got[0])


def test_shapes_of_a_step():
    f = F.Fit(*network((32, 16), torch.float32, 3), 6)
    bins = torch.zeros(6, dtype=torch.int32, device="cuda")
    for x, b in ((torch.zeros(1, 32), bins), (torch.zeros(6, 16), bins), (torch.zeros(6, 32), bins[:1])):
        with pytest.raises(ValueError):
            f.step(x.cuda(), b, 0.1)
