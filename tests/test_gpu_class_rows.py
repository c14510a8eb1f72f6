"""Rows of the classes' loss stand by themselves: what one row of x or of the table holds has no part in what another one's products give."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from test_gpu_classes import U, Reference, close, forward, host
from test_gpu_embed import BF16, F32, dev

pytestmark = pytest.mark.gpu


def gradients(x, e, b, ids, lse):
    dx, de, db = torch.empty_like(x), torch.empty_like(e), None if b is None else torch.empty_like(b)
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b, dbias_out=db)
    return dx, de, db


@pytest.mark.parametrize("size", [1.0e6, 1.0e15, -1.8e19, float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_without_a_class_may_hold_anything(dtype, size):
    """Padding rows beside rows that count, in the same 32: the loss, lse of the others and all gradients have the same bits as with zeros there."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    n, classes, d = 333, 150, 96
    x = torch.randn((n, d), generator=gen, device=dev()).to(dtype)
    e = (0.2 * torch.randn((classes, d), generator=gen, device=dev())).to(dtype)
    b = torch.randn(classes, generator=gen, device=dev())
    ids = torch.randint(0, classes, (n,), generator=gen, device=dev())
    padding = torch.arange(n, device=dev()) % 7 == 3
    padding[-9:] = True
    ids[padding] = -1
    x[padding] = 0.0
    loss, lse = forward(x, e, b, ids, n)
    want = gradients(x, e, b, ids, lse)
    x[padding] = size
    loss2, lse2 = forward(x, e, b, ids, n)
    assert torch.equal(loss, loss2) and torch.equal(lse[~padding], lse2[~padding])
    for got, w in zip(gradients(x, e, b, ids, lse2), want):
        assert torch.equal(got, w)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_the_table_that_are_taken_out_may_be_large(dtype):
    """A class with a bias of -inf has probability 0 whatever its row: 2^50 there leaves lse of all rows as it is, and the gradients right."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    n, classes, d = 200, 130, 64
    x = torch.randn((n, d), generator=gen, device=dev()).to(dtype)
    e = (0.2 * torch.randn((classes, d), generator=gen, device=dev())).to(dtype)
    b = torch.randn(classes, generator=gen, device=dev())
    out = torch.arange(classes, device=dev()) % 5 == 2
    b[out] = float("-inf")
    ids = torch.randint(0, classes // 5, (n,), generator=gen, device=dev()) * 5
    e[out] = 0.0
    loss, lse = forward(x, e, b, ids, n)
    ref = Reference(host(x), host(e), b.double().cpu().numpy(), ids.cpu().numpy(), dtype)
    want = ref.gradients(lse.double().cpu().numpy(), 1.0)
    e[out] = 2.0 ** 50
    loss2, lse2 = forward(x, e, b, ids, n)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    dx, de, db = gradients(x, e, b, ids, lse2)
    close(host(dx), *want["dx"], dtype)
    close(host(de), *want["dtable"], dtype)
    close(db.double().cpu().numpy(), *want["dbias"])
    assert not de[out].any()


def test_every_row_of_its_own_size():
    """Neighbouring rows from 2^-20 to 2^20, the table's rows the other way round, so that logits are of ordinary size: float rows enter the products
    as multiples of 2^-22 of each value or 2^-39 of their own largest.  Each gives d terms of three products and what they leave out, 8 u of each
    (u = 2^-24): 14 d u of the sum of absolute values at most, and the sum of the two in 32 bits 2 u |z|; exp and log take 10 u (1 + |z|) more."""
    rng = np.random.default_rng(8)
    n, d = 96, 64
    powers = 2.0 ** (20.0 * np.cos(np.arange(n) * 2.1))
    x = torch.from_numpy(rng.standard_normal((n, d)) * powers[:, None]).float().to(dev())
    for i in range(0, n, 7):                    # a table for one row at a time: logits of all rows would leave float32's range
        e = torch.from_numpy(rng.standard_normal((40, d)) / powers[i] * (2.0 ** np.linspace(-6, 0, 40))[:, None] * 0.5).float().to(dev())
        _, lse = forward(x, e, None, torch.full((n,), -1, device=dev()), n)
        xs, es = host(x)[i], host(e)
        z, size = es @ xs, np.abs(es) @ np.abs(xs)
        p = np.exp(z - z.max())
        want = z.max() + np.log(p.sum())
        assert abs(lse[i].item() - want) <= U * (14 * d * size.max() + 12 * (1 + np.abs(z).max())), (i, lse[i].item(), want)
