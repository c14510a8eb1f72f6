"""dz in the second products of the classes' gradients: what is kept of small ones."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from test_gpu_classes import host, put
from test_gpu_embed import BF16, F32, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [0, -10, -20, -30])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rare_classes_of_small_features(dtype, power):
    """Features and a table scaled by 2^-20 and the like, classes of probabilities down to e^-40: every row of dE is right relative to its own largest value,
    to 1e-4 for floats (sums of 200 terms, each right to 1e-5 and more) and 2^-7 for 16 bits (half a step, and dz)."""
    rng = np.random.default_rng(9)
    n, classes, d = 200, 300, 64
    x, e = (put(rng.standard_normal((rows, d)) * size * 2.0 ** power, dtype) for rows, size in ((n, 1.0), (classes, 0.2)))
    b = put(-40.0 * rng.random(classes))
    rare = torch.argsort(b)[:150]
    ids = torch.argsort(b, descending=True)[torch.from_numpy(rng.integers(0, 20, n)).to(dev())]         # no rare class has a row
    z = host(x) @ host(e).T + b.double().cpu().numpy()
    lse = put(np.log(np.exp(z).sum(1)))
    dx, de = torch.empty_like(x), torch.empty_like(e)
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b)
    dz = np.exp(z - lse.double().cpu().numpy()[:, None])
    dz[np.arange(n), ids.cpu().numpy()] -= 1.0
    for got, want in ((host(de), dz.T @ host(x) / n), (host(dx), dz @ host(e) / n)):
        worst = np.abs(got - want).max(1) / np.abs(want).max(1)
        assert worst.max() <= (1e-4 if dtype == F32 else 2.0 ** -7), (worst.max(), worst.argmax())
    assert bool((de[rare] != 0).any(1).all())
