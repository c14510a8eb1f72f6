"""Refusals of the embedding and tensor-list entry points, none of which reach the device."""
from array import array

import pytest

import paper_2603_27156_amd as gsr

P = 4096            # stands for a device address: nothing of it is read before the arguments are found wrong
OK, BAD, UNSUPPORTED, SMALL = gsr.GSR_OK, gsr.GSR_ERR_INVALID_ARG, gsr.GSR_ERR_UNSUPPORTED, gsr.GSR_ERR_WORKSPACE_TOO_SMALL


def lookup(table=P, vocab=10, ldt=8, table_dtype=0, ids=P, i64=0, n=4, d=8, c=2, layout=0, dtype=0, scale=1.0, x=P, ldx=8):
    return gsr.lib().gsr_embed_lookup(table, vocab, ldt, table_dtype, ids, i64, n, d, c, layout, dtype, scale, x, ldx, None)


def grad(ids=P, i64=0, n=5000, dx=P, ldx=8, d=8, c=2, layout=0, dtype=0, scale=1.0, vocab=10, out=P, ldt=8, ws=P, nbytes=1 << 24):
    return gsr.lib().gsr_embed_grad(ids, i64, n, dx, ldx, d, c, layout, dtype, scale, vocab, out, ldt, ws, nbytes, None)


SHAPES = [(dict(n=-1), BAD), (dict(n=2 ** 31), UNSUPPORTED), (dict(d=0), UNSUPPORTED), (dict(d=131_073, ldx=131_073, ldt=131_073), UNSUPPORTED),
          (dict(c=0), UNSUPPORTED), (dict(c=3), UNSUPPORTED), (dict(layout=2), BAD), (dict(ldx=7), BAD), (dict(layout=1, ldx=3), BAD),
          (dict(ldx=2 ** 31), BAD), (dict(vocab=0), BAD), (dict(vocab=2 ** 31 - 1), UNSUPPORTED), (dict(ldt=7), BAD), (dict(dtype=2), UNSUPPORTED),
          (dict(d=131_072, c=131_072, layout=1, ldx=1, ldt=131_072), UNSUPPORTED)]


@pytest.mark.parametrize("change,status", SHAPES + [(dict(table_dtype=-1), UNSUPPORTED), (dict(table=None), BAD), (dict(ids=None), BAD),
                                                    (dict(x=None), BAD), (dict(table=P + 2), BAD), (dict(x=P + 1, dtype=1), BAD),
                                                    (dict(ids=P + 4, i64=1), BAD)])
def test_lookup_refuses(change, status):
    assert lookup(**change) == status and gsr.gsr_last_error()


def test_lookup_of_nothing_is_done():
    assert lookup(n=0, table=None, ids=None, x=None) == OK


@pytest.mark.parametrize("change,status", SHAPES + [(dict(ids=None), BAD), (dict(dx=None), BAD), (dict(out=None), BAD), (dict(ws=None), BAD),
                                                    (dict(ws=P + 8), BAD), (dict(nbytes=100), SMALL), (dict(dx=P + 2), BAD), (dict(out=P + 1), BAD)])
def test_grad_refuses(change, status):
    assert grad(**change) == status and gsr.gsr_last_error()


def test_grad_workspace_is_monotonic_and_refuses_the_same_sizes():
    size = gsr.gsr_embed_grad_workspace
    assert size(0, 1, 1) == size(4096, 100, 64) == 0 < size(4097, 1, 1) <= size(100_000, 1, 1) <= size(100_000, 5_000, 1) <= size(100_000, 5_000, 256)
    assert size(1_000_000, 5_000, 256) < 1_000_000 * (20 + 256 // 8 + 2)
    for bad in ((-1, 1, 1), (2 ** 31, 1, 1), (1, 0, 1), (1, 2 ** 31 - 1, 1), (1, 1, 0), (1, 1, 131_073)):
        assert size(*bad) == 0
    need = size(5000, 10, 8)
    assert grad(nbytes=need - 1) == SMALL


@pytest.mark.parametrize("vocab", [97, 1_500, 50_021, 2 ** 22])
@pytest.mark.parametrize("d", [1, 3, 17, 32, 33, 64, 77, 256, 530, 1024, 4100, 131_072])
def test_grad_workspace_for_n_rows_serves_fewer(vocab, d):
    """Over sizes of every scale, and one by one around those where the sort takes longer stretches or the sums longer chunks."""
    size, most = gsr.gsr_embed_grad_workspace, 2 ** 31 - 1
    edges = {4096, 16_384, 32_768} | {(k << 20) // d for k in (16, 17, 32, 33, 64, 65, 128, 129, 256, 257)} | {k << 21 for k in (1, 2, 3, 8, 64)}
    ns = {int(1.03 ** i) for i in range(726)} | {e + i for e in edges for i in range(-2, 3)}
    before = 0
    for n in sorted(n for n in ns if 0 <= n <= most):
        now = size(n, vocab, d)
        assert before <= now <= n * (18 + 0.55 * d) + 64 * d + 2 ** 23, (n, before, now)
        before = now


def test_grad_takes_the_workspace_of_a_larger_graph():
    """What a call asks for is never more than what a call of more rows does: 69,631 rows of 256 take chunks of 16 rows, 69,632 of 32."""
    size = gsr.gsr_embed_grad_workspace
    assert size(69_632, 97, 256) >= size(69_631, 97, 256) > 8 * 69_631
    assert grad(n=69_631, d=256, ldx=256, ldt=256, vocab=97, nbytes=5_328_640) == SMALL        # enough for the chunks of 32 alone


class Lists:
    """Host arrays of addresses and sizes, one list per keyword; they live as long as this does."""

    def __init__(self, counts, **lists):
        self.arrays = {k: array("Q", v) for k, v in lists.items()}
        self.counts = array("q", counts)

    def __getitem__(self, k):
        return self.arrays[k].buffer_info()[0]

    @property
    def sizes(self):
        return self.counts.buffer_info()[0]


def norm(counts=(4, 4), g=(P, 2 * P), dtype=0, out=P, ws=P, nbytes=1 << 20, tensors=None):
    a = Lists(counts, g=g)
    return gsr.lib().gsr_grad_norm(a["g"], a.sizes, len(counts) if tensors is None else tensors, dtype, out, ws, nbytes, None)


def clip(counts=(4, 4), g=(P, 2 * P), dtype=0, max_norm=1.0, out=None, out_dtype=0, norm_out=None, ws=P, nbytes=1 << 20, tensors=None):
    a = Lists(counts, g=g, out=out or ())
    return gsr.lib().gsr_grad_clip(a["g"], a.sizes, len(counts) if tensors is None else tensors, dtype, max_norm, norm_out,
                                   a["out"] if out else None, out_dtype, ws, nbytes, None)


def adam(counts=(4, 4), w=(P, 2 * P), dw=(3 * P, 4 * P), m=(5 * P, 6 * P), v=(7 * P, 8 * P), dtype=0, norm=None, max_norm=1.0, t=1, beta1=0.9,
         beta2=0.999, tensors=None):
    a = Lists(counts, w=w, dw=dw, m=m, v=v)
    return gsr.lib().gsr_adam_update_list(a["w"], a["dw"], a["m"], a["v"], a.sizes, len(counts) if tensors is None else tensors, dtype, norm,
                                          max_norm, t, 1e-3, beta1, beta2, 1e-8, 0.0, None)


@pytest.mark.parametrize("change,status", [
    (dict(tensors=-1), BAD), (dict(counts=(4, -1)), BAD), (dict(counts=(2 ** 40, 1)), UNSUPPORTED), (dict(g=(P, 0)), BAD), (dict(g=(P, P + 2)), BAD),
    (dict(dtype=2), UNSUPPORTED), (dict(dtype=1, g=(P, P + 1)), BAD), (dict(out=None), BAD), (dict(out=P + 2), BAD), (dict(ws=None), BAD),
    (dict(ws=P + 4), BAD), (dict(nbytes=255), SMALL)])
def test_norm_refuses(change, status):
    assert norm(**change) == status and gsr.gsr_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(tensors=-1), BAD), (dict(counts=(4, -1)), BAD), (dict(g=(P, 0)), BAD), (dict(dtype=2), UNSUPPORTED), (dict(max_norm=-1.0), BAD),
    (dict(max_norm=float("inf")), BAD), (dict(max_norm=float("nan")), BAD), (dict(norm_out=P + 2), BAD), (dict(nbytes=255), SMALL),
    (dict(ws=None), BAD), (dict(out=(3 * P, 4 * P), out_dtype=2), UNSUPPORTED), (dict(out=(3 * P, 0)), BAD),
    # what is written lies over something else: the same tensor twice, a view of another, an output over a gradient or another output
    (dict(g=(P, P)), BAD), (dict(g=(P, P + 12)), BAD), (dict(g=(P + 12, P)), BAD), (dict(out=(P, 4 * P)), BAD), (dict(out=(3 * P, 3 * P + 12)), BAD),
    (dict(out=(3 * P, 2 * P + 12)), BAD), (dict(counts=(400, 4), out=(3 * P, 3 * P + 400)), BAD)])
def test_clip_refuses(change, status):
    assert clip(**change) == status and gsr.gsr_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(tensors=-1), BAD), (dict(counts=(-4, 4)), BAD), (dict(w=(P, 0)), BAD), (dict(dtype=-1), UNSUPPORTED), (dict(t=0), BAD), (dict(beta1=1.0), BAD),
    (dict(beta2=-0.1), BAD), (dict(norm=P, max_norm=-1.0), BAD), (dict(norm=P, max_norm=float("inf")), BAD), (dict(norm=P + 1), BAD),
    (dict(w=(P, P)), BAD), (dict(m=(P, 6 * P)), BAD), (dict(dw=(P, 4 * P)), BAD), (dict(v=(7 * P, 5 * P + 12)), BAD)])
def test_adam_refuses(change, status):
    assert adam(**change) == status and gsr.gsr_last_error()


# the norm and the workspace are written while tensors are read (P + 12: the last float of four at P), the norm of an update is read meanwhile
@pytest.mark.parametrize("call", [
    lambda: norm(out=P + 12, ws=16 * P), lambda: norm(out=2 * P, ws=16 * P), lambda: norm(out=16 * P, ws=2 * P), lambda: norm(out=16 * P, ws=P + 8),
    lambda: norm(out=16 * P, ws=2 * P - 256), lambda: norm(out=16 * P, ws=16 * P), lambda: norm(out=16 * P + 264, ws=16 * P),
    lambda: norm(dtype=1, out=P + 4, ws=16 * P), lambda: clip(norm_out=P, ws=16 * P), lambda: clip(norm_out=2 * P + 12, ws=16 * P), lambda: clip(ws=P),
    lambda: clip(out=(3 * P, 4 * P), norm_out=4 * P + 4, ws=16 * P), lambda: clip(out=(3 * P, 4 * P), ws=3 * P),
    lambda: clip(out=(3 * P, 4 * P), out_dtype=1, norm_out=3 * P + 4, ws=16 * P), lambda: clip(norm_out=16 * P + 8, ws=16 * P),
    lambda: adam(norm=P), lambda: adam(norm=2 * P + 12), lambda: adam(norm=5 * P + 4), lambda: adam(norm=8 * P)])
def test_a_norm_or_workspace_over_a_tensor_is_refused(call):
    assert call() == BAD and gsr.gsr_last_error()


def test_empty_lists_and_tensors():
    assert adam(tensors=0) == OK and adam(counts=(0, 0), w=(0, 0), dw=(0, 0), m=(0, 0), v=(0, 0)) == OK
    lib = gsr.lib()
    assert lib.gsr_grad_norm_workspace(None, 0) > 0 and lib.gsr_grad_norm_workspace(None, -1) == 0
    a = Lists((5, -1), g=())
    assert lib.gsr_grad_norm_workspace(a.sizes, 2) == 0


def test_an_update_with_a_norm_has_to_say_what_it_clips_to():
    torch = pytest.importorskip("torch")
    x = [torch.zeros(4)]
    with pytest.raises(TypeError, match="max_norm"):
        gsr.gsr_adam_update_list(x, x, x, x, 1, 1e-3, norm=torch.ones(1))


def test_lists_of_tensors_are_read_as_they_are():
    """The binding's helper on host tensors: what it refuses, and that it does so before an address is used."""
    torch = pytest.importorskip("torch")
    f, counts, which = gsr_marshal(), array("q", [0, 0]), array("q", [0])
    at = array("Q", [0, 0])

    def read(tensors, n=2, dtype=0, device=-1, compare=0):
        return f(tensors, n, device, dtype, compare, at.buffer_info()[0], counts.buffer_info()[0], which.buffer_info()[0]), which[0]

    a, b = torch.zeros(4), torch.zeros(3, 2)
    for good in ([a, b], (a, b), [torch.nn.Parameter(a), b]):
        assert read(good) == (3, 0)                          # host tensors: not on the GPU
    assert read([a]) == (1, 0) and read(iter([a, b])) == (1, 0) and read([1, a]) == (2, 0) and read([a.to_sparse(), a]) == (2, 0)
    assert at == array("Q", [0, 0])
    with pytest.raises((TypeError, RuntimeError, AssertionError)):
        gsr.gsr_grad_norm([a, b], a)
    assert read([], n=0) == (0, 0)


def gsr_marshal():
    import ctypes as C
    f = C.PyDLL(gsr.MARSHAL_PATH).gsr_marshal_list
    f.restype = C.c_int
    f.argtypes = [C.py_object, C.c_int64, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
    return f
