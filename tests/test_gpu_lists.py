"""Gradient norm, clipping and Adam over lists of tensors against their definitions in 64 bits.

The norm is summed in 64 bits and rounded once (2^-24; 2^-23 leaves room for the sums of 2^-53 each).  A clipped gradient is the product with a
coefficient in 64 bits, rounded once in float32 (2^-24, subnormal results 2^-150) and, for 16 bits, again (2^-8, 2^-134).  Adam's float32
arithmetic is bit for bit that of gsr_adam_update where nothing is clipped (and 1 - beta comes to the same number); where something is, the clipped gradient is rounded twice more
(the coefficient, from a rounded norm, and the product: under 2^-22 of the gradient)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import optim
import paper_2603_27156_amd as gsr
from paper_2603_27156_amd import synth
from gpu_util import Case, assert_close

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
GUARD = -7.0


def dev():
    return torch.device("cuda:0")


SIZES = {
    "one": [1], "none": [], "empty": [0, 0], "scalars": [1] * 7, "around": [4095, 0, 4096, 4097, 1, 8192, 3], "large": [3_000_017],
    "many": [1 + (i * 37) % 300 for i in range(1000)], "mixed": [5, 100_003, 1, 4096, 70_000, 0, 33],
}


def make(sizes, dtype, values, gap=1, offset=1):
    """Tensors of these sizes in one buffer of GUARD, `gap` elements between them, the first `offset` elements in: (buffer, tensors)."""
    buffer = torch.full((offset + sum(sizes) + gap * len(sizes),), GUARD, dtype=dtype, device=dev())
    out, at = [], offset
    for k in sizes:
        out.append(buffer[at:at + k])
        at += k + gap
    for t, v in zip(out, values.split(sizes)) if sizes else ():
        t.copy_(v)
    return buffer, out


def flat(tensors, dtype=torch.float64):
    return torch.cat([t.to(dtype).cpu() for t in tensors]) if tensors else torch.zeros(0, dtype=dtype)


def gaps_untouched(buffer, sizes, gap=1, offset=1):
    mask, at = torch.ones_like(buffer, dtype=torch.bool), offset
    for k in sizes:
        mask[at:at + k] = False
        at += k + gap
    return bool((buffer[mask] == GUARD).all())


def randn(k, seed=0):
    return torch.randn(k, generator=torch.Generator("cuda").manual_seed(seed), device=dev())


def norm_of(tensors):
    out = torch.full((1,), GUARD, device=dev())
    gsr.gsr_grad_norm(tensors, out)
    return float(out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
@pytest.mark.parametrize("offset", [0, 1])
def test_norm(sizes, dtype, offset):
    _, g = make(sizes, dtype, randn(sum(sizes)) * 3, offset=offset, gap=offset)
    want = float(flat(g).norm())
    assert abs(norm_of(g) - want) <= 2.0 ** -23 * want


def test_norm_of_numbers_whose_squares_no_float_holds():
    for scale in (1e30, 1e-30, 2.0 ** -149, 1.0):
        g = [(randn(5000) * scale).contiguous(), randn(77, 1) * scale]
        want = float(flat(g).norm())
        assert want > 0 and abs(norm_of(g) - want) <= max(2.0 ** -23 * want, 2.0 ** -149)
    big = torch.full((100,), 3e38, device=dev())
    assert norm_of([big]) == float("inf")                    # the norm itself is beyond float32
    assert norm_of([torch.tensor([1.0, float("inf")], device=dev())]) == float("inf")
    assert np.isnan(norm_of([torch.tensor([1.0, float("nan"), float("inf")], device=dev())]))


CLIP_TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]


def clip_close(got, want, dtype):
    step, low = (2.0 ** -24, 2.0 ** -150) if dtype == F32 else (2.0 ** -8 + 2.0 ** -24, 2.0 ** -134)
    return bool(((got - want).abs() <= step * want.abs() * (1 + 2.0 ** -20) + low).all())


@pytest.mark.parametrize("dtype,out_dtype", CLIP_TYPES)
@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
def test_clip_into_other_tensors(sizes, dtype, out_dtype):
    buffer, g = make(sizes, dtype, randn(sum(sizes)) * 3)
    out_buffer, out = make(sizes, out_dtype, torch.zeros(sum(sizes), device=dev()), gap=3, offset=2)
    before, exact = buffer.clone(), flat(g)
    norm = torch.empty(1, device=dev())
    for max_norm in (0.75, 1e6, 0.0):
        gsr.gsr_grad_clip(g, max_norm, norm, out=out)
        size = float(exact.norm())
        assert abs(float(norm) - size) <= 2.0 ** -23 * size
        assert clip_close(flat(out), exact * min(1.0, float(np.float32(max_norm)) / (size + 1e-6)), out_dtype)
        assert torch.equal(buffer, before) and gaps_untouched(out_buffer, sizes, 3, 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
def test_clip_in_place(sizes, dtype):
    buffer, g = make(sizes, dtype, randn(sum(sizes)) * 3)
    before, exact = buffer.clone(), flat(g)
    gsr.gsr_grad_clip(g, 1e6)
    assert torch.equal(buffer, before)                       # already short enough: the same bits
    gsr.gsr_grad_clip(g, 0.75)
    assert clip_close(flat(g), exact * min(1.0, 0.75 / (float(exact.norm()) + 1e-6)), dtype)
    assert gaps_untouched(buffer, sizes)
    gsr.gsr_grad_clip(g, 0.0)
    assert bool((flat(g) == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_clip_of_what_is_not_finite(dtype):
    g = [randn(5000).to(dtype), torch.tensor([2.0, float("inf")], dtype=dtype, device=dev())]
    norm = torch.zeros(1, device=dev())
    gsr.gsr_grad_clip(g, 1.0, norm)
    assert float(norm) == float("inf") and bool((g[0] == 0).all()) and float(g[1][0]) == 0 and bool(g[1][1].isnan())
    g = [randn(5000).to(dtype), torch.tensor([2.0, float("nan")], dtype=dtype, device=dev())]
    gsr.gsr_grad_clip(g, 1.0, norm)
    assert bool(norm.isnan()) and all(bool(t.isnan().all()) for t in g)


ADAM = dict(t=7, lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=1e-2)
EXACT = dict(ADAM, beta1=0.875, beta2=0.96875)               # 1 - beta is a float32 whatever way it is rounded


def adam_lists(sizes, dw_dtype, seed=0):
    k = sum(sizes)
    w, m = make(sizes, F32, randn(k, seed)), make(sizes, F32, randn(k, seed + 2) * 0.1, gap=2)
    v, g = make(sizes, F32, randn(k, seed + 3).square(), offset=3), make(sizes, dw_dtype, randn(k, seed + 1) * 2)
    return w, g, m, v


@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
def test_adam_list_is_adam_on_every_tensor(sizes):
    (wb, w), (gb, g), (mb, m), (vb, v) = adam_lists(sizes, F32)
    alone = [[t.clone() for t in x] for x in (w, g, m, v)]
    guards = wb.clone(), gb.clone()
    gsr.gsr_adam_update_list(w, g, m, v, **EXACT)
    for a, b, c, d in zip(*alone):
        gsr.gsr_adam_update(a, b, c, d, **EXACT)
    for got, want in zip((w, g, m, v), alone):
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert gaps_untouched(wb, sizes) and gaps_untouched(mb, sizes, 2) and gaps_untouched(vb, sizes, 1, 3) and torch.equal(gb, guards[1])
    # a norm that needs no clipping changes nothing either
    again = adam_lists(sizes, F32)
    gsr.gsr_adam_update_list(*(x[1] for x in again), norm=torch.full((1,), 3.0, device=dev()), max_norm=4.0, **EXACT)
    assert torch.equal(again[0][0], wb) and torch.equal(again[2][0], mb) and torch.equal(again[3][0], vb)


@pytest.mark.parametrize("dw_dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", SIZES.values(), ids=SIZES)
def test_clipped_adam(sizes, dw_dtype):
    (wb, w), (gb, g), (mb, m), (vb, v) = adam_lists(sizes, dw_dtype)
    w0, g0, m0, v0 = (flat(x).numpy() for x in (w, g, m, v))
    norm = torch.zeros(1, device=dev())
    gsr.gsr_grad_norm(g, norm)
    gsr.gsr_adam_update_list(w, g, m, v, norm=norm, max_norm=0.5, **ADAM)
    c = min(1.0, 0.5 / (float(np.sqrt((g0 ** 2).sum())) + 1e-6))
    b1, b2, lr, eps, wd = (ADAM[k] for k in ("beta1", "beta2", "lr", "eps", "weight_decay"))
    rw, rm, rv = optim.adam(w0, c * g0, m0, v0, ADAM["t"], lr, b1, b2, eps, wd)
    assert_close("w", flat(w).numpy(), rw)
    assert_close("m", flat(m).numpy(), rm)
    assert_close("v", flat(v).numpy(), rv)
    assert np.array_equal(flat(g).numpy(), g0)


def test_first_step_with_state_of_zeros_keeps_every_digit():
    """m and v of the first step are (1 - beta) g and (1 - beta2) g^2: three roundings each (1 - beta, and one or two products)."""
    g = randn(5000, 4)
    w, m, v = torch.zeros_like(g), torch.zeros_like(g), torch.zeros_like(g)
    gsr.gsr_adam_update_list([w], [g], [m], [v], 1, 1e-3)
    x = g.double()
    assert bool(((m.double() - 0.1 * x).abs() <= 3 * 2.0 ** -24 * (0.1 * x).abs()).all())
    assert bool(((v.double() - 0.001 * x * x).abs() <= 3 * 2.0 ** -24 * 0.001 * x * x).all())


def test_captured_calls_of_two_graphs_on_one_workspace():
    lists = []
    for i, name in enumerate(("mixed", "many")):
        _, g = make(SIZES[name], F32, randn(sum(SIZES[name]), i))
        lists.append((g, torch.zeros(1, device=dev())))
    ws = torch.empty(max(gsr.gsr_grad_norm_workspace(g) for g, _ in lists), dtype=torch.uint8, device=dev())
    side = torch.cuda.Stream()
    graphs = []
    for g, norm in lists:
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            gsr.gsr_grad_clip([t.clone() for t in g], 0.5, norm, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            gsr.gsr_grad_clip(g, 0.5, norm, workspace=ws)
        graphs.append(graph)
    for step in range(3):
        for (g, norm), graph in zip(lists, graphs):
            for i, t in enumerate(g):
                t.copy_(randn(t.numel(), 100 * step + i))
            want, size = [t.clone() for t in g], torch.zeros(1, device=dev())
            gsr.gsr_grad_clip(want, 0.5, size)
            ws.random_()
            norm.fill_(GUARD)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(norm, size) and all(torch.equal(a, b) for a, b in zip(g, want))


def test_binding_refuses_what_does_not_fit():
    a, b = torch.zeros(8, device=dev()), torch.zeros(8, device=dev())
    one = torch.zeros(1, device=dev())
    for bad in (lambda: gsr.gsr_grad_norm([a, b.bfloat16()], one), lambda: gsr.gsr_grad_norm([a[::2]], one), lambda: gsr.gsr_grad_norm([a.cpu()], one),
                lambda: gsr.gsr_grad_norm([a.double()], one), lambda: gsr.gsr_grad_norm([a], b), lambda: gsr.gsr_grad_norm([a], one.double()),
                lambda: gsr.gsr_grad_clip([a], 1.0, out=[b[:4]]), lambda: gsr.gsr_grad_clip([a], 1.0, out=[b, b]),
                lambda: gsr.gsr_adam_update_list([a], [b], [b], [], t=1, lr=1.0)):
        with pytest.raises((AssertionError, TypeError)):
            bad()
    for bad in (lambda: gsr.gsr_grad_clip([a, a], 1.0), lambda: gsr.gsr_grad_clip([a, a[2:4]], 1.0), lambda: gsr.gsr_grad_clip([a], -1.0),
                lambda: gsr.gsr_grad_clip([a], 1.0, out=[a]), lambda: gsr.gsr_adam_update_list([a], [b], [a], [b], t=1, lr=1.0),
                lambda: gsr.gsr_grad_norm([a], one, workspace=one)):
        with pytest.raises(gsr.GsrError):
            bad()
    for bad in (lambda: gsr.gsr_grad_norm([a, 1], one), lambda: gsr.gsr_grad_norm([a, None], one), lambda: gsr.gsr_grad_norm(a, one),
                lambda: gsr.gsr_grad_norm(iter([a]), one), lambda: gsr.gsr_grad_clip([a], 1.0, out=[b[::2]]),
                lambda: gsr.gsr_grad_clip([a, b], 1.0, out=[b.clone()])):
        with pytest.raises((AssertionError, TypeError)):
            bad()
    gsr.gsr_grad_norm([a, a], one)                           # only read: a tensor may count twice
    gsr.gsr_grad_norm((torch.nn.Parameter(a), b.view(2, 4)), one)


# ---- long lists ------------------------------------------------------------------------------------------------------
# The norm takes chunks of 4,096 elements, one partial sum per workgroup, 16,384 workgroups a launch at most.  Clipping adds up to 1,024 partial sums
# by itself; above that, and for the norm always, a launch of 1,024 threads does, each four at a time, again and again above 4,096.  A chunk that
# was left out would be one of 33,000 equal shares of the sum of squares at least, more than 2^-17 of the norm, where 2^-23 is asked for.
CHUNK = 4096
LONG = {
    "1023 chunks": [1023 * CHUNK], "1024 chunks": [1000 * CHUNK, 24 * CHUNK], "1025 chunks": [1024 * CHUNK + 1], "1024 and a launch": [1] * 1024,
    "1025 in six launches": [1] * 1025, "1800 in four launches": [2 * CHUNK + 77] * 600, "4099 chunks": [5, 4096 * CHUNK, CHUNK + 3],
    "9000 chunks": [9000 * CHUNK - 7], "16390 chunks of one launch": [3 * CHUNK, 16_384 * CHUNK + 17, 2 * CHUNK],
    "33000 chunks in two launches": [9] * 190 + [16_500 * CHUNK, 16_310 * CHUNK],
}
long_lists = pytest.mark.parametrize("sizes", LONG.values(), ids=LONG)


def long_list(sizes, dtype):
    """(buffer, tensors, the same values in float64 in one piece)"""
    buffer, g = make(sizes, dtype, randn(sum(sizes)) * 3)
    return buffer, g, torch.cat(g).double()


@pytest.mark.parametrize("dtype", [F32, BF16])
@long_lists
def test_norm_of_long_lists(sizes, dtype):
    _, g, exact = long_list(sizes, dtype)
    want = float(exact.square().sum().sqrt())
    assert abs(norm_of(g) - want) <= 2.0 ** -23 * want


@pytest.mark.parametrize("dtype,out_dtype", [(F32, None), (BF16, None), (F32, BF16), (BF16, F32)])
@long_lists
def test_clip_of_long_lists(sizes, dtype, out_dtype):
    buffer, g, exact = long_list(sizes, dtype)
    before, size, norm = buffer.clone(), float(exact.square().sum().sqrt()), torch.zeros(1, device=dev())
    out_buffer, out, to = buffer, g, None
    if out_dtype is not None:
        out_buffer, out = make(sizes, out_dtype, torch.zeros(sum(sizes), device=dev()), gap=3, offset=2)
        to = out
    for max_norm in (2.0 * size, 0.75):
        gsr.gsr_grad_clip(g, max_norm, norm, out=to)
        assert abs(float(norm) - size) <= 2.0 ** -23 * size
        assert clip_close(torch.cat(out).double(), exact * min(1.0, 0.75 / (size + 1e-6) if max_norm < size else 1.0), out[0].dtype)
        if to is not None or max_norm > size:
            assert torch.equal(buffer, before)
    assert gaps_untouched(out_buffer, sizes, *((1, 1) if to is None else (3, 2)))


@pytest.mark.parametrize("dw_dtype", [F32, BF16])
@long_lists
def test_clipped_adam_of_long_lists(sizes, dw_dtype):
    (wb, w), (gb, g), (mb, m), (vb, v) = adam_lists(sizes, dw_dtype)
    w0, g0, m0, v0 = (torch.cat(x).double() for x in (w, g, m, v))
    size, norm = float(g0.square().sum().sqrt()), torch.zeros(1, device=dev())
    gsr.gsr_grad_norm(g, norm)
    gsr.gsr_adam_update_list(w, g, m, v, norm=norm, max_norm=0.5, **ADAM)
    gk = g0 * (0.5 / (size + 1e-6)) + ADAM["weight_decay"] * w0
    m1 = ADAM["beta1"] * m0 + (1 - ADAM["beta1"]) * gk
    v1 = ADAM["beta2"] * v0 + (1 - ADAM["beta2"]) * gk * gk
    step = (m1 / (1 - ADAM["beta1"] ** ADAM["t"])) / ((v1 / (1 - ADAM["beta2"] ** ADAM["t"])).sqrt() + ADAM["eps"])
    for name, got, want in (("w", w, w0 - ADAM["lr"] * step), ("m", m, m1), ("v", v, v1)):
        low = 1e-5 * min(1.0, float(want.square().mean().sqrt()))
        assert bool(((torch.cat(got).double() - want).abs() <= low + 1e-4 * want.abs()).all()), name
    assert gaps_untouched(wb, sizes) and gaps_untouched(mb, sizes, 2) and gaps_untouched(vb, sizes, 1, 3)


# ---- a training step with all of them, as a program makes it ---------------------------------------------------------
class Training:
    """Nodes with tokens of a small vocabulary: lookup, gsr_step, gradient of the table, norm, clipped Adam."""

    def __init__(self, n=1201, l=3, vocab=23, layout=gsr.GSR_LAYOUT_GROUP_PLANAR):
        w = synth.scaled(synth.workload(1), n, l=l)
        self.case = c = Case(w, 0, layout)
        c.gcfg.k = c.ocfg.k = w.d // w.c                     # all columns kept: no selection that a rounding could turn
        rng = np.random.default_rng(3)
        self.vocab, self.scale, self.lr, self.max_norm = vocab, float(np.float32(np.sqrt(w.d))), 2e-3, 0.02
        self.ids_host = rng.integers(-1, vocab, n)
        f32 = dict(dtype=F32, device=dev())
        groups = (w.c, n, w.d // w.c) if layout == gsr.GSR_LAYOUT_GROUP_PLANAR else (n, w.d)
        self.ids = torch.from_numpy(self.ids_host).to(dev())
        self.table_host = (rng.standard_normal((vocab, w.d)) / self.scale).astype(np.float32)
        self.W_host = np.ascontiguousarray(c.inp.weights[:l])
        self.params = [torch.from_numpy(x.copy()).to(dev()) for x in (self.table_host, self.W_host, c.inp.w_out)] + [torch.zeros(1, **f32)]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.m, self.v = [torch.zeros_like(p) for p in self.params], [torch.zeros_like(p) for p in self.params]
        self.x0, self.dx0 = torch.zeros(groups, **f32), torch.zeros(groups, **f32)
        self.loss, self.norm, self.target = torch.zeros(1, **f32), torch.zeros(1, **f32), torch.from_numpy(c.inp.target).to(dev())
        self.ws = torch.empty(gsr.gsr_workspace_size(c.gg, c.gcfg)[1], dtype=torch.uint8, device=dev())
        self.ews = torch.empty(gsr.gsr_embed_grad_workspace(n, vocab, w.d), dtype=torch.uint8, device=dev())
        self.nws = torch.empty(gsr.gsr_grad_norm_workspace(self.grads), dtype=torch.uint8, device=dev())

    def gradients(self):
        table, W, w_out, b = self.params
        dtable, dW, dw, db = self.grads
        gsr.gsr_embed_lookup(table, self.ids, self.x0, self.scale)
        gsr.gsr_step(self.case.gg, self.case.gcfg, self.x0, W, w_out, b, self.target, self.loss, dW, dw, db, dx0_out=self.dx0, workspace=self.ws)
        gsr.gsr_embed_grad(self.ids, self.dx0, dtable, self.scale, workspace=self.ews)
        gsr.gsr_grad_norm(self.grads, self.norm, workspace=self.nws)

    def step(self, t):
        self.gradients()
        gsr.gsr_adam_update_list(self.params, self.grads, self.m, self.v, t, self.lr, norm=self.norm, max_norm=self.max_norm)

    def reference(self, table):
        """Loss and gradients of the oracle for this table (float64 behind the float32 plane)."""
        known = self.ids_host >= 0
        x0 = np.where(known[:, None], table[np.clip(self.ids_host, 0, None)].astype(np.float32) * np.float32(self.scale), np.float32(0))
        ref = oracle.step(self.case.og, self.case.ocfg, self.W_host.shape[0], x0, self.W_host, self.case.inp.w_out, 0.0, self.case.inp.target)
        dtable = np.zeros(table.shape)
        np.add.at(dtable, self.ids_host[known], np.asarray(ref["dX0"], dtype=np.float64)[known] * self.scale)
        return ref, dtable


@pytest.mark.parametrize("layout", [gsr.GSR_LAYOUT_ROW_MAJOR, gsr.GSR_LAYOUT_GROUP_PLANAR])
def test_training_step_against_the_oracle(layout):
    s = Training(layout=layout)
    s.gradients()
    ref, dtable = s.reference(s.table_host)
    assert np.isclose(float(s.loss), ref["loss"], rtol=1e-4)
    assert_close("dtable", s.grads[0].cpu().numpy(), dtable)
    # dW, dw and db are gsr_step's, which has its own tests: what follows takes them as they are
    g = [dtable, np.asarray(ref["dW"], dtype=np.float64), np.asarray(ref["dwout"], dtype=np.float64), np.array([ref["dbout"]], dtype=np.float64)]
    norm = np.sqrt(sum((x ** 2).sum() for x in g))
    assert np.isclose(float(s.norm), norm, rtol=1e-4) and norm > s.max_norm       # so the update is clipped
    got = [x.double().cpu().numpy() for x in s.grads]
    norm = float(np.sqrt(sum((x ** 2).sum() for x in got)))
    assert abs(float(s.norm) - norm) <= 2.0 ** -23 * norm
    c = s.max_norm / (norm + 1e-6)
    before = [p.double().cpu().numpy() for p in s.params]
    gsr.gsr_adam_update_list(s.params, s.grads, s.m, s.v, 1, s.lr, norm=s.norm, max_norm=s.max_norm)
    for i, p in enumerate(s.params):
        w, m, v = optim.adam(before[i], c * got[i], 0.0, 0.0, 1, s.lr)
        assert_close("m", s.m[i].cpu().numpy(), m)
        assert_close("v", s.v[i].cpu().numpy(), v)
        assert_close("w", p.cpu().numpy(), w)


@pytest.mark.parametrize("layout", [gsr.GSR_LAYOUT_ROW_MAJOR, gsr.GSR_LAYOUT_GROUP_PLANAR])
def test_every_gradient_of_a_training_step_against_the_oracle(layout):
    """Tensor by tensor: the weights of every block against its largest entry (sums of 1,201 products that partly cancel, as the audits of whole
    layers take them), the head element by element, the bias as a number."""
    s = Training(layout=layout)
    s.gradients()
    ref, dtable = s.reference(s.table_host)
    got = [x.double().cpu().numpy() for x in s.grads]
    assert_close("dtable", got[0], dtable)
    dW = np.asarray(ref["dW"], dtype=np.float64)
    worst = np.abs(got[1] - dW).max(axis=(2, 3)) / np.abs(dW).max(axis=(2, 3))
    assert worst.shape == dW.shape[:2] and (worst <= 1e-4).all(), worst
    assert_close("dw", got[2], ref["dwout"])
    assert np.isclose(got[3][0], ref["dbout"], rtol=1e-4, atol=1e-7)


def test_table_gradient_against_differences():
    """All columns kept, no RMS scale: the loss is a quadratic function of the table, of which a central difference in the oracle's double
    arithmetic gives the derivative but for the rounding of the plane to float32 (2^-24 of entries that move by 2^-6 of their size)."""
    s = Training(n=301, l=1)
    s.case.gcfg.norm, s.case.ocfg.norm, s.case.ocfg.sm = gsr.GSR_NORM_NONE, oracle.NORM_NONE, oracle.STORE_F64
    s.gradients()
    got = s.grads[0].double().cpu().numpy()
    rng = np.random.default_rng(1)
    for _ in range(4):
        direction = rng.standard_normal(s.table_host.shape)
        h = 2.0 ** -6
        up, down = (s.table_host + h * direction).astype(np.float32), (s.table_host - h * direction).astype(np.float32)
        slope = s.reference(up)[0]["loss"] - s.reference(down)[0]["loss"]
        moved = (up.astype(np.float64) - down.astype(np.float64))
        want = (got * moved).sum()
        size = np.abs(got * moved).sum()
        assert abs(slope - want) <= 1e-4 * size, (slope, want, size)


def test_captured_training_step_replays_like_the_eager_one():
    Training().step(1)                                       # every kernel has run once
    eager, played = Training(), Training()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        played.step(3)
    for _ in range(4):
        eager.step(3)                                        # a captured step keeps its counter
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert float(eager.loss) == float(played.loss) and torch.equal(eager.norm, played.norm)
        for a, b in zip(eager.params + eager.grads + eager.m + eager.v, played.params + played.grads + played.m + played.v):
            assert torch.equal(a, b)


def test_clip_then_update_is_the_clipped_update():
    """gsr_grad_clip followed by gsr_adam_update on every tensor, as an earlier program has it, against the list form: the clipped gradients
    differ by four roundings (norm, coefficient, a product on each side), Adam's v by twice that and two products on each side: 12 of 2^-24."""
    a, b = Training(), Training()
    a.gradients()
    gsr.gsr_grad_clip(a.grads, a.max_norm)
    for p, g, m, v in zip(a.params, a.grads, a.m, a.v):
        gsr.gsr_adam_update(p, g, m, v, 1, a.lr, 0.875, 0.96875)
    b.gradients()
    gsr.gsr_adam_update_list(b.params, b.grads, b.m, b.v, 1, b.lr, 0.875, 0.96875, norm=b.norm, max_norm=b.max_norm)
    for x, y in zip(a.m + a.v, b.m + b.v):
        assert bool(((x - y).abs() <= 2.0 ** -20 * x.abs() + 1e-30).all())
