"""Refusals of the softmax cross entropy over many classes, none of which reach the device."""
import pytest

import paper_2603_27156_amd as gsr

P = 4096            # stands for a device address: nothing of it is read before the arguments are found wrong
BAD, UNSUPPORTED, SMALL = gsr.GSR_ERR_INVALID_ARG, gsr.GSR_ERR_UNSUPPORTED, gsr.GSR_ERR_WORKSPACE_TOO_SMALL


def loss(x=P, ldx=8, n=4, d=8, c=2, layout=0, dtype=0, table=P, classes=10, ldt=8, bias=P, ids=P, i64=0, out=P, lse=P, ws=P, nbytes=1 << 24):
    return gsr.lib().gsr_class_loss(x, ldx, n, d, c, layout, dtype, table, classes, ldt, bias, ids, i64, out, lse, ws, nbytes, None)


def grad(x=P, ldx=8, n=4, d=8, c=2, layout=0, dtype=0, table=P, classes=10, ldt=8, bias=P, ids=P, i64=0, lse=P, scale=1.0, dx=P, lddx=8, dt=P, lddt=8,
         db=P, ws=P, nbytes=1 << 24):
    return gsr.lib().gsr_class_grad(x, ldx, n, d, c, layout, dtype, table, classes, ldt, bias, ids, i64, lse, scale, dx, lddx, dt, lddt, db, ws, nbytes,
                                    None)


SHARED = [(dict(n=-1), BAD), (dict(n=2 ** 28), UNSUPPORTED), (dict(classes=0), BAD), (dict(classes=2 ** 28), UNSUPPORTED), (dict(d=0), UNSUPPORTED),
          (dict(d=513, ldx=513, ldt=513), UNSUPPORTED), (dict(c=0), UNSUPPORTED), (dict(c=3), UNSUPPORTED), (dict(layout=2), BAD), (dict(dtype=2), UNSUPPORTED),
          (dict(ldx=7), BAD), (dict(layout=1, ldx=3), BAD), (dict(ldx=2 ** 31), BAD), (dict(ldt=7), BAD), (dict(ldt=2 ** 31), BAD), (dict(x=None), BAD),
          (dict(table=None), BAD), (dict(ids=None), BAD), (dict(x=P + 2), BAD), (dict(table=P + 1, dtype=1), BAD), (dict(bias=P + 2), BAD), (dict(ids=P + 4, i64=1), BAD),
          (dict(lse=None), BAD), (dict(lse=P + 2), BAD), (dict(ws=None), BAD), (dict(ws=P + 8), BAD), (dict(nbytes=100), SMALL)]


@pytest.mark.parametrize("change,status", SHARED + [(dict(out=None), BAD), (dict(out=P + 1), BAD)])
def test_loss_refuses(change, status):
    assert loss(**change) == status and gsr.gsr_last_error()


@pytest.mark.parametrize("change,status", SHARED + [(dict(dx=None, dt=None, db=None), BAD), (dict(lddx=7), BAD), (dict(lddx=2 ** 31), BAD), (dict(lddt=7), BAD),
                                                    (dict(lddt=2 ** 31), BAD), (dict(dx=P + 2), BAD), (dict(dt=P + 2), BAD), (dict(db=P + 2), BAD)])
def test_grad_refuses(change, status):
    assert grad(**change) == status and gsr.gsr_last_error()


def test_workspaces():
    lib = gsr.lib()
    for size in (lib.gsr_class_loss_workspace, lib.gsr_class_grad_workspace):
        assert 0 < size(0, 1, 1, 0) <= size(2_000, 40, 64, 0)
        # some copies of x and of the table, and nothing of the order n * classes
        assert size(1_000_000, 50_000, 256, 1) < 8 * 1_050_000 * 256 * 4
        for bad in ((-1, 1, 1, 0), (2 ** 28, 1, 1, 0), (1, 0, 1, 0), (1, 2 ** 28, 1, 0), (1, 1, 0, 0), (1, 1, 513, 0), (1, 1, 1, 2)):
            assert size(*bad) == 0
    assert loss(nbytes=lib.gsr_class_loss_workspace(4, 10, 8, 0) - 1) == SMALL and grad(nbytes=lib.gsr_class_grad_workspace(4, 10, 8, 0) - 1) == SMALL


@pytest.mark.parametrize("d,dtype", [(1, 0), (64, 0), (256, 1), (384, 0), (512, 1)])
def test_a_workspace_serves_fewer_rows_and_classes(d, dtype):
    sizes = sorted({int(1.13 ** i) for i in range(140)} | {255, 256, 257, 32_768, 65_536, 131_072, 131_073})
    for size in (gsr.lib().gsr_class_loss_workspace, gsr.lib().gsr_class_grad_workspace):
        for other in (1, 33, 4_099, 50_021, 1_000_000):
            rows = [size(n, other, d, dtype) for n in sizes]
            classes = [size(other, n, d, dtype) for n in sizes]
            assert rows == sorted(rows) and classes == sorted(classes)
