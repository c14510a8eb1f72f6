"""Graphs of a batch stand by themselves: what one of them holds has no part in the others."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from test_gpu_embed import BF16, F32, dev
from test_gpu_norm import U, Reference, close, host, put

pytestmark = pytest.mark.gpu


def forward(x, ptr, groups, **kw):
    y = torch.zeros_like(x)
    mean, rstd = (torch.empty((len(ptr) - 1, groups), device=dev()) for _ in range(2))
    gsr.gsr_group_norm(x, y, mean, rstd, graph_ptr=ptr, **kw)
    return y, mean, rstd


@pytest.mark.parametrize("value", [1.0e7, -1.0e9, 1.0e15])
@pytest.mark.parametrize("where", [0, 5, 63])
@pytest.mark.parametrize("d,planes,groups,dtype", [(64, 0, 4, F32), (64, 2, 2, BF16), (77, 0, 7, F32), (385, 0, 1, BF16), (5, 0, 5, F32)])
def test_a_large_value_stays_in_its_graph(d, planes, groups, dtype, where, value):
    """One value of the first graph far from all others, its very first one among the places: the other graphs' results have the same bits as without it,
    and its own mean and rstd are right.  Sums in 64 bits from one of the graph's own values: of count values they leave the variance 4 count 2^-53 of
    itself at most; then one rounding each."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    n = 64 * 5 + 3
    ptr = torch.tensor([3, 3 + 64, 3 + 64 * 2, 3 + 64 * 2, 3 + 64 * 5], device=dev())
    x = torch.randn((n, d) if not planes else (planes, n, d // planes), generator=gen, device=dev()).to(dtype)
    y, mean, rstd = forward(x, ptr, groups)
    x[..., 3 + where, 0] = value
    y2, mean2, rstd2 = forward(x, ptr, groups)
    assert torch.equal(y2[..., 67:, :], y[..., 67:, :]) and torch.equal(mean2[1:], mean[1:]) and torch.equal(rstd2[1:], rstd[1:])
    ref = Reference(host(x), ptr.tolist(), groups, None, None, "none")
    allowed = U + 4 * 2.0 ** -53 * 64 * d
    assert (np.abs(rstd2.double().cpu().numpy() - ref.rstd) <= 2 * allowed * ref.rstd).all()
    assert (np.abs(mean2.double().cpu().numpy() - ref.mean) <= 2 * allowed * np.abs(host(x)).max()).all()


@pytest.mark.parametrize("far", [1.0e6, 1.0e9])
def test_graphs_of_very_different_size(far):
    """Graphs of values around 0, `far` and -far, each with a spread of a few units in the last place of its mean: mean and rstd of each."""
    rng = np.random.default_rng(2)
    sizes, centres = [40, 70, 33, 200], [far, 0.0, -far, 0.3 * far]
    spread = max(1.0, far * 2.0 ** -20)
    rows = np.concatenate([c + spread * rng.standard_normal((s, 32)) for s, c in zip(sizes, centres)])
    ptr = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), device=dev())
    x = put(rows)
    _, mean, rstd = forward(x, ptr, 2)
    ref = Reference(host(x), ptr.tolist(), 2, None, None, "none")
    close(mean.double().cpu().numpy(), ref.mean, 2 * U * np.abs(ref.mean))
    close(rstd.double().cpu().numpy(), ref.rstd, 2 * U * ref.rstd)
