"""Graphs of a batch stand by themselves: what one of them holds, and how many of them are empty, has no part in the others."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from test_gpu_embed import BF16, F32, dev
from test_gpu_norm import ACTS, U, Reference, close, host, put

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


def empty_runs(kind, empty):
    """First rows of graphs in 300 rows, `empty` of them without a row at one offset inside a chunk of rows."""
    at = {"middle": [0, 103] + [103] * empty + [203, 290], "padded": [0, 103, 203] + [203] * empty, "front": [11] * (empty + 1) + [103, 203],
          "many": list(np.repeat([0, 5, 6, 7, 8, 103, 104, 203, 299], max(1, empty // 9)))}[kind]
    return torch.tensor(at, dtype=torch.int32, device=dev())


@pytest.mark.parametrize("kind", ["middle", "padded", "front", "many"])
@pytest.mark.parametrize("empty", [1, 2, 63, 64, 65, 4_000])
@pytest.mark.parametrize("d,groups,dtype,act", [(64, 4, F32, "silu"), (77, 7, BF16, "relu")])
def test_empty_graphs_anywhere(d, groups, dtype, act, empty, kind):
    rng = np.random.default_rng(empty)
    ptr = empty_runs(kind, empty)
    x, dy = put(rng.standard_normal((300, d)), dtype), put(rng.standard_normal((300, d)), dtype)
    gamma, beta = put(1.0 + 0.3 * rng.standard_normal(d)), put(0.3 * rng.standard_normal(d))
    y, mean, rstd = forward(x, ptr, groups, gamma=gamma, beta=beta, act=ACTS[act])
    g64, b64 = gamma.double().cpu().numpy(), beta.double().cpu().numpy()
    ref = Reference(host(x), ptr.tolist(), groups, g64, b64, act)
    close(mean.double().cpu().numpy(), ref.mean, 2 * U * np.abs(ref.mean) + 2.0 ** -50)
    close(rstd.double().cpu().numpy(), ref.rstd, 2 * U * ref.rstd)
    ref = Reference(host(x), ptr.tolist(), groups, g64, b64, act, mean.double().cpu().numpy(), rstd.double().cpu().numpy())
    close(host(y), *ref.forward(), dtype)
    dx, dgamma, dbeta = torch.zeros_like(x), torch.empty(d, device=dev()), torch.empty(d, device=dev())
    gsr.gsr_group_norm_grad(dy, mean, rstd, dx, x=x, gamma=gamma, beta=beta, act=ACTS[act], graph_ptr=ptr, dgamma_out=dgamma, dbeta_out=dbeta)
    want, off = ref.backward(host(dy))
    close(host(dx), want["dx"], off["dx"], dtype)
    close(dgamma.double().cpu().numpy(), want["dgamma"], off["dgamma"])
    close(dbeta.double().cpu().numpy(), want["dbeta"], off["dbeta"])
    spare = torch.ones(300, dtype=torch.bool, device=dev())
    spare[ptr[0]:ptr[-1]] = False
    assert not y[spare].any() and not dx[spare].any()


@pytest.mark.parametrize("kind", ["middle", "padded", "front"])
def test_empty_graphs_are_not_walked_one_by_one(kind):
    """A captured step has room for a fixed number of graphs, and most may be empty.  Two million of them at one offset: both directions end within 50 ms (a
    wave that steps through them, two loads that depend on each other a graph, takes some two seconds; their statistics are 16 MB)."""
    ptr = empty_runs(kind, 2_000_000)
    x = torch.randn((300, 64), device=dev())
    dx = torch.empty_like(x)
    ws = torch.empty(gsr.gsr_group_norm_workspace(x, 1, ptr), dtype=torch.uint8, device=dev())
    took = []
    for _ in range(2):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        y, mean, rstd = forward(x, ptr, 1, workspace=ws)
        gsr.gsr_group_norm_grad(y, mean, rstd, dx, x=x, graph_ptr=ptr, workspace=ws)
        end.record()
        end.synchronize()
        took.append(start.elapsed_time(end))
    assert min(took) <= 50.0, took


@pytest.mark.parametrize("d,groups,dtype,rows", [(1, 1, F32, 8192), (3, 3, F32, 8192), (4, 1, F32, 4096), (8, 1, BF16, 4096), (24, 24, BF16, 1024), (64, 2, F32, 1024),
                                                 (256, 32, BF16, 512)])
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_rows_about_the_single_launch(d, groups, dtype, rows, more):
    """A single graph of as many rows as one launch takes, one fewer and one more."""
    rng = np.random.default_rng(d)
    n = rows + more
    x, dy = put(rng.standard_normal((n, d)) + 3.0, dtype), put(rng.standard_normal((n, d)), dtype)
    y, (mean, rstd) = torch.empty_like(x), (torch.empty((1, groups), device=dev()) for _ in range(2))
    gsr.gsr_group_norm(x, y, mean, rstd, act=ACTS["silu"])
    ref = Reference(host(x), [0, n], groups, None, None, "silu")
    close(mean.double().cpu().numpy(), ref.mean, 2 * U * np.abs(ref.mean))
    close(rstd.double().cpu().numpy(), ref.rstd, 2 * U * ref.rstd)
    ref = Reference(host(x), [0, n], groups, None, None, "silu", mean.double().cpu().numpy(), rstd.double().cpu().numpy())
    close(host(y), *ref.forward(), dtype)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(d, device=dev()), torch.empty(d, device=dev())
    gsr.gsr_group_norm_grad(dy, mean, rstd, dx, x=x, act=ACTS["silu"], dgamma_out=dgamma, dbeta_out=dbeta)
    want, off = ref.backward(host(dy))
    close(host(dx), want["dx"], off["dx"], dtype)
    close(dgamma.double().cpu().numpy(), want["dgamma"], off["dgamma"])
    close(dbeta.double().cpu().numpy(), want["dbeta"], off["dbeta"])
