"""Refusals of group norm and of checkpoints in 8 bits, none of which reach the device."""
import pytest

import paper_2603_27156_amd as gsr

P = 4096            # stands for a device address: nothing of it is read before the arguments are found wrong
OK, BAD, UNSUPPORTED, SMALL = gsr.GSR_OK, gsr.GSR_ERR_INVALID_ARG, gsr.GSR_ERR_UNSUPPORTED, gsr.GSR_ERR_WORKSPACE_TOO_SMALL


def norm(x=P, ldx=8, n=4, d=8, c=2, layout=0, dtype=0, ptr=P, i64=0, graphs=3, groups=2, gamma=P, beta=P, eps=1e-5, act=0, y=2 * P, ldy=8, mean=P,
         rstd=P, codes=None, scales=None, ws=P, nbytes=1 << 24):
    return gsr.lib().gsr_group_norm(x, ldx, n, d, c, layout, dtype, ptr, i64, graphs, groups, gamma, beta, eps, act, y, ldy, mean, rstd, codes, scales,
                                    ws, nbytes, None)


def grad(dy=P, lddy=8, x=2 * P, ldx=8, codes=None, scales=None, n=4, d=8, c=2, layout=0, dtype=0, ptr=P, i64=0, graphs=3, groups=2, mean=P, rstd=P,
         gamma=P, beta=P, act=0, dx=3 * P, lddx=8, dgamma=P, dbeta=P, ws=P, nbytes=1 << 24):
    return gsr.lib().gsr_group_norm_grad(dy, lddy, x, ldx, codes, scales, n, d, c, layout, dtype, ptr, i64, graphs, groups, mean, rstd, gamma, beta, act,
                                         dx, lddx, dgamma, dbeta, ws, nbytes, None)


def save(x=P, ldx=8, n=4, d=8, c=2, layout=0, dtype=0, codes=P, scales=P):
    return gsr.lib().gsr_checkpoint_save(x, ldx, n, d, c, layout, dtype, codes, scales, None)


def load(codes=P, scales=P, n=4, d=8, c=2, layout=0, dtype=0, x=P, ldx=8):
    return gsr.lib().gsr_checkpoint_load(codes, scales, n, d, c, layout, dtype, x, ldx, None)


PLANES = [(dict(n=-1), BAD), (dict(n=2 ** 31), UNSUPPORTED), (dict(d=0), UNSUPPORTED), (dict(d=131_073), UNSUPPORTED), (dict(c=0), UNSUPPORTED),
          (dict(c=3), UNSUPPORTED), (dict(layout=2), BAD), (dict(dtype=2), UNSUPPORTED), (dict(d=8192, c=8192, layout=1), UNSUPPORTED)]
X = [(dict(x=None), BAD), (dict(x=P + 2), BAD), (dict(x=P + 1, dtype=1), BAD), (dict(ldx=7), BAD), (dict(layout=1, ldx=3, d=8), BAD),
     (dict(ldx=2 ** 31), BAD)]
NORM = [(dict(graphs=-1), BAD), (dict(graphs=2 ** 31), UNSUPPORTED), (dict(ptr=None), BAD), (dict(ptr=None, graphs=0), BAD), (dict(ptr=P + 2), BAD),
        (dict(ptr=P + 4, i64=1), BAD), (dict(groups=0), UNSUPPORTED), (dict(groups=3), UNSUPPORTED), (dict(groups=16), UNSUPPORTED), (dict(act=3), UNSUPPORTED),
        (dict(act=-1), UNSUPPORTED), (dict(mean=None), BAD), (dict(rstd=None), BAD), (dict(mean=P + 2), BAD), (dict(gamma=P + 1), BAD),
        (dict(beta=P + 2), BAD), (dict(ws=None), BAD), (dict(ws=P + 8), BAD), (dict(nbytes=255), SMALL), (dict(codes=P), BAD), (dict(scales=P), BAD)]


@pytest.mark.parametrize("change,status", PLANES + X + NORM + [
    (dict(y=None), BAD), (dict(y=P + 2), BAD), (dict(ldy=7), BAD), (dict(eps=0.0), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("inf")), BAD),
    (dict(eps=float("nan")), BAD), (dict(y=P, ldy=9), BAD), (dict(codes=P + 2, scales=P), BAD), (dict(codes=P, scales=P + 2), BAD)])
def test_norm_refuses(change, status):
    assert norm(**change) == status and gsr.gsr_last_error()


@pytest.mark.parametrize("change,status", PLANES + X + [c for c in NORM if "codes" not in c[0] and "scales" not in c[0]] + [
    (dict(dy=None), BAD), (dict(dy=P + 2), BAD), (dict(lddy=7), BAD), (dict(dx=None), BAD), (dict(dx=P + 2), BAD), (dict(lddx=7), BAD),
    (dict(dx=P, lddx=9), BAD), (dict(dgamma=P + 2), BAD), (dict(dbeta=P + 1), BAD), (dict(codes=P, scales=P), BAD), (dict(x=None, codes=P), BAD),
    (dict(x=None, scales=P), BAD), (dict(x=None, codes=P + 2, scales=P), BAD)])
def test_norm_grad_refuses(change, status):
    assert grad(**change) == status and gsr.gsr_last_error()


@pytest.mark.parametrize("change,status", PLANES + X + [(dict(codes=None), BAD), (dict(scales=None), BAD), (dict(codes=P + 1), BAD), (dict(scales=P + 2), BAD)])
def test_checkpoints_refuse(change, status):
    assert save(**change) == status and gsr.gsr_last_error()
    assert load(**change) == status and gsr.gsr_last_error()


def test_nothing_to_do():
    assert norm(n=0, x=None, y=None, graphs=0, mean=None, rstd=None) == OK
    assert norm(n=4, graphs=0, mean=None, rstd=None) == OK
    assert save(n=0, x=None, codes=None, scales=None) == OK and load(n=0, x=None, codes=None, scales=None) == OK


def test_workspace():
    def size(n, graphs, d, c=1, layout=0, dtype=0, groups=1):
        return gsr.lib().gsr_group_norm_workspace(n, graphs, d, c, layout, dtype, groups)
    assert 0 < size(0, 1, 64) <= size(2000, 1, 64) < 1 << 20 and size(1_000_000, 1, 256, 4, 1, 0, 4) < 32 << 20
    assert size(1_000_000, 4_000, 256, groups=32) < 64 << 20
    need = size(4, 3, 8, 2, 0, 0, 2)
    assert norm(nbytes=need - 1) == SMALL
    for bad in ((-1, 1, 64), (2 ** 31, 1, 64), (4, -1, 64), (4, 2 ** 31, 64), (4, 1, 0), (4, 1, 131_073), (4, 1, 64, 3), (4, 1, 64, 1, 2), (4, 1, 64, 1, 0, 2),
                (4, 1, 64, 1, 0, 0, 0), (4, 1, 64, 1, 0, 0, 3), (4, 1, 64, 1, 0, 0, 128)):
        assert size(*bad) == 0
    assert norm(n=2 ** 31 - 1, d=64, ldx=64, ldy=64, graphs=2 ** 31 - 1, groups=64) == UNSUPPORTED         # more sums than can be named


@pytest.mark.parametrize("d,c,layout,dtype,groups", [(1, 1, 0, 0, 1), (64, 2, 1, 0, 2), (256, 1, 0, 1, 32), (77, 1, 0, 0, 7), (384, 2, 1, 1, 6), (131_072, 1, 0, 0, 8)])
def test_a_workspace_serves_fewer_rows_and_graphs(d, c, layout, dtype, groups):
    size = gsr.lib().gsr_group_norm_workspace
    slabs = -(-d // 256)
    sizes = sorted({int(1.07 ** i) for i in range(300)} | {8192 * k // slabs + i for k in (1, 8, 32, 64, 1024) for i in range(-2, 3)})
    sizes = [n for n in sizes if 0 <= n < 2 ** 31]
    for other in (1, 300):
        rows = [size(n, other, d, c, layout, dtype, groups) for n in sizes]
        graphs = [size(other, n, d, c, layout, dtype, groups) for n in sizes]
        assert rows == sorted(rows) and graphs == sorted(graphs)
