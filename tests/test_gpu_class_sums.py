"""The sums of the classes' loss over long sides: sums of whole numbers, in which nothing can be lost without being seen, and the small probabilities beside
a large one."""
import math

import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from test_gpu_classes import U, forward
from test_gpu_embed import BF16, F32, dev

pytestmark = pytest.mark.gpu


def whole(shape, most, seed, dtype):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=gen, device=dev()).to(dtype)


def grad(x, e, ids, lse, **kw):
    dx, de, db = torch.empty_like(x), torch.empty_like(e), torch.empty(len(e), device=dev())
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, dbias_out=db, **kw)
    return dx, de, db


SIZES = [(70_001, 23, 40), (70_001, 70, 64), (131_001, 5, 12), (33, 50_021, 48), (3, 131_101, 16), (2_050, 4_099, 200), (300, 2_000, 384), (65, 1_111, 512)]


@pytest.mark.parametrize("n,classes,d", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_row_is_lost_in_the_gradients(n, classes, d, dtype):
    """Whole numbers below 2^24 in every sum, so that float32 sums are exact in any order, and scale = rows, so that nothing is divided: with x = 0 every
    exp(z - lse) is 1 for lse = 0 and dx = sum E - E_t; with E = 0 dE = sum x - sum of the class's x.  An infinite lse leaves -1 at the class
    alone.  One rounding of the output, which torch's own conversion gives too."""
    ids = torch.randint(0, classes, (n,), generator=torch.Generator(device="cuda").manual_seed(n), device=dev())
    ids[::11] = -1
    known = ids >= 0
    count = float(known.sum())
    zero, far = torch.zeros(n, device=dev()), torch.full((n,), float("inf"), device=dev())
    own = torch.bincount(ids[known], minlength=classes).double()

    most = 3 if classes > 100_000 else 15
    e, x = whole((classes, d), most, 1, dtype), torch.zeros((n, d), dtype=dtype, device=dev())
    dx, de, db = grad(x, e, ids, zero, scale=count)
    want = (e.double().sum(0) - e.double()[ids.clamp(min=0)]) * known[:, None]
    assert torch.equal(dx, want.to(dtype)) and not de.any() and torch.equal(db, (known.sum() - own).float())
    dx, de, db = grad(x, e, ids, far, scale=count)
    assert torch.equal(dx, (-e.double()[ids.clamp(min=0)] * known[:, None]).to(dtype)) and not de.any() and torch.equal(db, (-own).float())

    x, e = whole((n, d), 15, 2, dtype), torch.zeros((classes, d), dtype=dtype, device=dev())
    rows = x.double() * known[:, None]
    mine = torch.zeros((classes, d), dtype=torch.float64, device=dev()).index_add_(0, ids.clamp(min=0), rows)
    dx, de, db = grad(x, e, ids, zero, scale=count)
    assert torch.equal(de, (rows.sum(0) - mine).to(dtype)) and not dx.any() and torch.equal(db, (known.sum() - own).float())
    dx, de, db = grad(x, e, ids, far, scale=count)
    assert torch.equal(de, (-mine).to(dtype)) and not dx.any() and torch.equal(db, (-own).float())


@pytest.mark.parametrize("n,classes,d", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_class_is_lost_in_the_loss(n, classes, d, dtype):
    """Logits of 0: lse = log(classes), the loss the same.  The sum is exact; the logarithm of 32 bits is off by 2 u of itself, and so are the roundings."""
    x, e = torch.zeros((n, d), dtype=dtype, device=dev()), whole((classes, d), 15, 3, dtype)
    ids = torch.randint(0, classes, (n,), generator=torch.Generator(device="cuda").manual_seed(n), device=dev())
    loss, lse = forward(x, e, None, ids, n)
    want = math.log(classes)
    assert bool(((lse.double() - want).abs() <= 4 * U * want).all()) and abs(loss.item() - want) <= 4 * U * want


def learnt(classes, gap, spread, seed):
    """Logits of one row as whole multiples of 2^-10: one of them `gap` above a tail of this spread."""
    rng = np.random.default_rng(seed)
    z = np.round(rng.standard_normal(classes) * spread * 1024.0) / 1024.0
    z[classes // 3] = gap
    return z


@pytest.mark.parametrize("gap", [16.0, 16.5, 17.0, 18.0, 25.0])
@pytest.mark.parametrize("spread", [0.0, 0.3, 2.0])
@pytest.mark.parametrize("n,classes", [(65_600, 50_021), (5_000, 50_021), (70, 50_021), (1, 50_021), (65_600, 33)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_probabilities_beside_a_large_one(dtype, n, classes, gap, spread):
    """A row that is nearly learnt: the loss is log(1 + the tail), which is right relative to itself.  The logits are the bias, exact; x = 0.  Every term is
    exp of an exact difference w: off by (3 |w| + 2) u (difference, product, function); what was summed before the largest
    is multiplied by exp of its way, and where the maximum grew before that by at most all of |w| and 4 more steps, as much again; then the join's
    parts as much a third time, log 2 u and the loss u.  With |w| <= gap + 5 spreads: 9 (gap + 5 spread) + 40 u relative.  A lane's 8 terms of a tile are added
    in pairs of pairs of 32 bits, off by 3 u of their sum, and all these sums together are 1 + the tail, the largest's 1 among them (its neighbours of the tile
    are added to it): 3 u of log's argument, which is 3 u of the loss, absolute."""
    z = learnt(classes, gap, spread, 7)
    tail = np.exp(np.delete(z, classes // 3) - gap).sum()
    want = math.log1p(tail)
    x, e = torch.zeros((n, 8), dtype=dtype, device=dev()), torch.ones((classes, 8), dtype=dtype, device=dev())
    b = torch.from_numpy(z).float().to(dev())
    ids = torch.full((n,), classes // 3, device=dev())
    loss, lse = forward(x, e, b, ids, n)
    relative = U * (9 * (gap + 5 * spread) + 40)
    assert abs(loss.item() - want) <= relative * want + 3 * U, (loss.item() / want - 1, relative)
    assert bool(((lse.double() - (gap + want)).abs() <= relative * want + 3 * U + U * (gap + want)).all())
    # From the kernel's own lse the probabilities of a row add up to 1, within lse's rounding (u |lse|), exp's (3 |w| + 4) u and dbias' own, u each
    db = torch.empty(classes, device=dev())
    gsr.gsr_class_grad(x, e, ids, lse, bias=b, dbias_out=db)
    off = U * (gap + want + 3) + relative * want + U * (np.exp(z - gap) * (3 * np.abs(z - gap) + 8)).sum()
    assert abs(db.double().sum().item()) <= off, (db.double().sum().item(), off)
    others = torch.arange(classes, device=dev()) != classes // 3
    share = db.double()[others].sum().item()
    assert abs(share - tail / (1 + tail)) <= share * (U * (3 * (gap + 5 * spread) + 11 + gap) + relative), share


@pytest.mark.parametrize("top", [2.0 ** 26, 2.0 ** 33, 2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_of_any_size(dtype, top):
    """Logits far above 2^24: exp of the difference from the largest, whatever its size."""
    x = torch.zeros((70, 32), dtype=dtype, device=dev())
    x[:, 0] = 2.0 ** 50 if top > 2.0 ** 40 else 2.0 ** 13
    e = torch.zeros((300, 32), dtype=dtype, device=dev())
    e[:, 0] = torch.linspace(-1.0, 1.0, 300, device=dev()).to(dtype).abs() * (top / x[0, 0].item())
    e[150, 0] = 1.41015625 * top / x[0, 0].item()
    largest = e[150, 0].item() * x[0, 0].item()                 # (of what the table's type makes of it)
    ids = torch.full((70,), 150, device=dev())
    loss, lse = forward(x, e, None, ids, 70)
    assert bool((lse == largest).all()) and loss.item() == 0.0
    dx, de, _ = grad(x, e, ids, lse)
    assert not dx.any() and not de.any()


def test_classes_in_order_of_their_logits():
    """The largest logit grows with every class, by little: what was summed before is multiplied again and again, and lse must not drift.  The reference
    follows the largest only where it is left behind by more than 1, 30 times here: 30 (2 + 1.5) u and the way, 3 * 30 u; 20 u besides."""
    classes, n = 50_021, 65_600
    b = torch.linspace(-15.0, 15.0, classes, device=dev())
    for z in (b, b.flip(0)):
        _, lse = forward(torch.zeros((n, 8), device=dev()), torch.ones((classes, 8), device=dev()), z, torch.full((n,), -1, device=dev()), n)
        want = torch.logsumexp(z.double(), 0)
        assert bool(((lse.double() - want).abs() <= U * (215 + want.abs())).all()), (lse.double() - want).abs().max().item() / U
