"""Softmax cross entropy over many classes and its gradient against the definitions in 64 bits.

u = 2^-24.  A sum of k terms on the matrix cores is off by at most 2 k u times the sum of absolute values (whether its additions round or
truncate).  Logits: 16-bit values give d terms; floats three products of pieces each, 3 d terms (bounded here by six), and what the pieces and the product of
the smaller ones leave out is below 2^-21 = 8 u of each value, or 2^-38 of the largest in 32 rows.  exp(z - l) by base 2: u |z - l| for the difference, 2 u |z - l| for the product, 2 u for the function.  lse: T tiles of a lane
have 8 additions each, and the running maximum is exchanged at most T times (2 u each, and 3 u of the way it goes).  dz: one rounding, and with
16-bit planes a relative 2^-8 more; then sums over all classes or rows, their parts joined (64 at most), and three roundings.  A 16-bit
output adds half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from test_gpu_embed import BF16, F32, GUARD, dev, make_ids, plane, rows_of, untouched

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def terms(dtype, k):
    return 2 * k if dtype == BF16 else 2 * 6 * k + 8


class Reference:
    """Loss, lse and gradients in float64 with bounds of the errors of float32 results, before they are rounded to 16 bits."""

    def __init__(self, x, e, b, ids, dtype):
        self.x, self.e, self.b, self.dtype = x, e, b, dtype
        n, d = x.shape
        self.t = np.where((ids >= 0) & (ids < len(e)), ids, -1)
        self.known = self.t >= 0
        self.count = int(self.known.sum())
        self.z = x @ e.T + b
        finite_b = np.where(np.isfinite(b), np.abs(b), 0.0)
        self.z_off = (terms(dtype, d) + 4) * U * (np.abs(x) @ np.abs(e).T + finite_b)
        self.small_x, self.small_e = (self.smallest(v) if dtype == F32 else np.zeros((len(v), 1)) for v in (x, e))
        self.z_off += self.small_x * np.abs(e).sum(1) + (self.small_e * np.abs(x).sum(1)).T
        top = self.z.max(1, keepdims=True) if n else np.zeros((0, 1))
        w = np.exp(self.z - top)
        self.lse = top[:, 0] + np.log(w.sum(1))
        p = w / w.sum(1, keepdims=True)
        way = np.where(p > 0, np.abs(np.where(p > 0, self.z, 0.0) - top), 0.0)
        low = np.where(np.isfinite(self.z), self.z, np.inf).min(1) if n else np.zeros(0)
        tiles = -(-len(e) // 32)
        self.lse_off = (p * (self.z_off + U * (3 * way + 2))).sum(1) + U * (10 * tiles + 8 + 3 * (top[:, 0] - low) + 2 * np.abs(self.lse))

    @staticmethod
    def smallest(v):
        """2^-38 of the largest value of every 32 rows, for each of them."""
        out = np.zeros((len(v), 1))
        for a in range(0, len(v), 32):
            out[a:a + 32] = 2.0 ** -38 * np.abs(v[a:a + 32]).max()
        return out

    def loss(self):
        """(loss, bound)."""
        if not self.count:
            return 0.0, 0.0
        at = self.z[self.known, self.t[self.known]]
        value = (self.lse[self.known] - at).sum() / self.count
        off = (self.lse_off[self.known] + self.z_off[self.known, self.t[self.known]]).sum() / self.count
        return value, off + 2 * U * abs(value)

    def gradients(self, lse, scale):
        """With lse as given (rounded)."""
        k = scale / max(1, self.count)
        p = np.exp(self.z - lse[:, None]) * self.known[:, None]
        way = np.where(p > 0, np.abs(np.where(p > 0, self.z, 0.0) - lse[:, None]), 0.0)
        off = p * (self.z_off + U * (3 * way + 4))
        dz = p.copy()
        dz[np.nonzero(self.known)[0], self.t[self.known]] -= 1.0
        off += 2 * U * np.abs(dz)
        bias = dz.sum(0) * k, off.sum(0) * abs(k) + 8 * U * (np.abs(dz)).sum(0) * abs(k)
        rounded = off + (2.0 ** -8 * (np.abs(dz) + off) if self.dtype == BF16 else 0.0)

        def product(dz, rounded, other, small, length):
            size = np.abs(dz) @ np.abs(other)
            off = rounded @ np.abs(other) + (terms(self.dtype, length) + 64 + 4) * U * size
            if self.dtype == F32 and dz.size:       # what pieces leave out: of the streamed rows, and of dz, 2^-36 of the largest product with a streamed tile
                off += np.abs(dz) @ np.broadcast_to(small, other.shape)
                tops = 2.0 ** 38 * small[:, 0]
                off += 2.0 ** -34 * (np.abs(dz) * tops).max(1, keepdims=True) * len(other)
            return dz @ other * k, off * abs(k)

        x = np.where(self.known[:, None], self.x, 0.0)
        return dict(dx=product(dz, rounded, self.e, self.small_e, len(self.e)), dtable=product(dz.T, rounded.T, x, self.smallest(x), len(self.x)), dbias=bias)


def close(got, want, off, dtype=F32):
    allowed = off + (np.abs(want) + off) * (2.0 ** -8 if dtype == BF16 else 0.0) + 2.0 ** -140
    worst = np.abs(got - want) - allowed
    assert got.shape == want.shape and (got.size == 0 or worst.max() <= 0.0), (worst.max(), np.abs(got - want).max(), np.isnan(got).sum())


def host(t):
    return rows_of(t).double().cpu().numpy()


def put(a, dtype=F32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(dev())


CASES = [
    # n, classes, d, c, dtype, ids, kind, pad, offset, bias
    (1, 1, 1, 0, F32, torch.int32, "one", 0, 0, True),
    (1, 1, 64, 2, BF16, torch.int64, "one", 0, 0, False),
    (1, 1000, 64, 0, F32, torch.int64, "mixed", 0, 0, True),
    (1, 50_021, 128, 0, BF16, torch.int32, "one", 0, 0, True),
    (2, 3, 3, 0, F32, torch.int32, "distinct", 2, 1, True),
    (17, 33, 32, 0, BF16, torch.int32, "mixed", 0, 0, True),
    (31, 5, 33, 0, F32, torch.int32, "mixed", 1, 3, False),
    (33, 257, 77, 0, BF16, torch.int64, "common", 3, 1, True),
    (64, 64, 64, 2, F32, torch.int32, "common", 0, 0, True),
    (100, 300, 100, 0, F32, torch.int64, "mixed", 0, 0, True),
    (129, 40, 192, 3, BF16, torch.int32, "mixed", 0, 0, True),
    (257, 1031, 192, 2, F32, torch.int32, "mixed", 4, 2, True),
    (300, 97, 256, 4, F32, torch.int32, "common", 0, 0, True),
    (300, 4_099, 256, 8, BF16, torch.int32, "mixed", 8, 8, True),
    (513, 700, 384, 2, F32, torch.int64, "common", 0, 0, True),
    (513, 700, 300, 0, BF16, torch.int32, "mixed", 0, 0, False),
    (70_001, 23, 64, 2, F32, torch.int32, "mixed", 0, 0, True),
    (70_001, 23, 40, 0, BF16, torch.int64, "mixed", 0, 0, True),
    (200, 333, 512, 2, F32, torch.int32, "mixed", 0, 0, True),
    (200, 333, 512, 8, BF16, torch.int32, "mixed", 0, 0, True),
    (65, 130, 511, 0, F32, torch.int32, "mixed", 1, 0, True),
    (65, 130, 511, 0, BF16, torch.int32, "mixed", 1, 1, True),
    (3_000, 20, 64, 2, F32, torch.int32, "common", 0, 0, True),
    (40_000, 33, 32, 0, BF16, torch.int64, "mixed", 0, 0, True),
    (70_000, 2, 24, 2, F32, torch.int32, "mixed", 0, 0, True),
    (2_111, 3_001, 40, 0, F32, torch.int32, "distinct", 0, 0, True),
    (300, 64, 48, 0, F32, torch.int32, "unknown", 0, 0, True),
]


def inputs(n, classes, d, c, dtype, ids_type, kind, pad, offset, bias):
    rng = np.random.default_rng(n + 7 * classes + d)
    _, x = plane(n, d, c, dtype, torch.from_numpy(rng.standard_normal((n, d))), pad, offset)
    _, e = plane(classes, d, 0, dtype, torch.from_numpy(rng.standard_normal((classes, d)) * 2.0 / np.sqrt(d)), pad, offset)
    b = rng.standard_normal(classes).astype(np.float32) if bias else None
    if bias and classes > 8:
        b[classes // 2] = -np.inf                      # a class taken out
    ids = make_ids(kind, n, classes, rng)
    if bias and classes > 8:
        ids = np.where(ids == classes // 2, 0, ids)
    ref = Reference(host(x), host(e), np.zeros(classes) if b is None else b.astype(np.float64), ids, dtype)
    return x, e, put(b), torch.from_numpy(ids).to(ids_type).to(dev()), ref


def forward(x, e, b, ids, n, **kw):
    loss, lse = torch.full((1,), GUARD, device=dev()), torch.full((n,), GUARD, device=dev())
    gsr.gsr_class_loss(x, e, ids, loss, lse, bias=b, **kw)
    return loss, lse


@pytest.mark.parametrize("n,classes,d,c,dtype,ids_type,kind,pad,offset,bias", CASES)
def test_loss(n, classes, d, c, dtype, ids_type, kind, pad, offset, bias):
    x, e, b, ids, ref = inputs(n, classes, d, c, dtype, ids_type, kind, pad, offset, bias)
    loss, lse = forward(x, e, b, ids, n)
    close(lse.double().cpu().numpy(), ref.lse, ref.lse_off)
    value, off = ref.loss()
    assert abs(loss.item() - value) <= off, (loss.item(), value, off)


@pytest.mark.parametrize("n,classes,d,c,dtype,ids_type,kind,pad,offset,bias", CASES)
def test_gradient(n, classes, d, c, dtype, ids_type, kind, pad, offset, bias):
    x, e, b, ids, ref = inputs(n, classes, d, c, dtype, ids_type, kind, pad, offset, bias)
    lse = put(ref.lse)
    dx_buffer, dx = plane(n, d, c, dtype, None, pad, offset)
    de_buffer, de = plane(classes, d, 0, dtype, None, pad, offset)
    db = torch.full((classes,), GUARD, device=dev())
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b, dbias_out=db, scale=1.5)
    want = ref.gradients(lse.double().cpu().numpy(), 1.5)
    close(host(dx), *want["dx"], dtype)
    close(host(de), *want["dtable"], dtype)
    close(db.double().cpu().numpy(), *want["dbias"])
    assert untouched(dx_buffer, dx) and untouched(de_buffer, de)
    # one at a time: the same bits
    for name, t in (("dx_out", dx), ("dtable_out", de), ("dbias_out", db)):
        alone = torch.full_like(t, GUARD) if t.is_contiguous() else plane(n if name == "dx_out" else classes, d, c if name == "dx_out" else 0, dtype, None, pad, offset)[1]
        gsr.gsr_class_grad(x, e, ids, lse, bias=b, scale=1.5, **{name: alone})
        assert torch.equal(alone, t), name


def test_gradient_against_differences():
    """Along random directions, against differences of the loss in 64 bits."""
    rng = np.random.default_rng(3)
    x, e, b, ids, ref = inputs(50, 37, 24, 0, F32, torch.int32, "mixed", 0, 0, False)
    b = put(rng.standard_normal(37))
    _, lse = forward(x, e, b, ids, 50)
    dx, de, db = torch.empty_like(x), torch.empty_like(e), torch.empty_like(b)
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b, dbias_out=db, scale=2.0)
    at = [host(x), host(e), b.double().cpu().numpy()]
    for i, got in enumerate((dx, de, db)):
        v = rng.standard_normal(at[i].shape)

        def loss(h):
            moved = list(at)
            moved[i] = moved[i] + h * v
            return 2.0 * Reference(*moved, ids.cpu().numpy(), F32).loss()[0]
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        along = got.double().cpu().numpy() * v
        # differences: third derivatives times h^2, below 1e-8; the kernel: 1e-5 of every term
        assert abs(along.sum() - slope) <= 1e-5 * np.abs(along).sum() + 1e-7, i


def test_large_logits_stay_finite():
    """Logits of hundreds: the maximum goes up from tile to tile, and down."""
    for sign in (1.0, -1.0):
        x = torch.full((70, 32), 1.0, device=dev())
        e = torch.zeros((500, 32), device=dev())
        e[:, 0] = sign * torch.linspace(-900.0, 900.0, 500, device=dev())
        ids = torch.arange(70, device=dev()) * 7
        loss, lse = forward(x, e, None, ids, 70)
        ref = Reference(host(x), host(e), np.zeros(500), ids.cpu().numpy(), F32)
        close(lse.double().cpu().numpy(), ref.lse, ref.lse_off)
        dx = torch.empty_like(x)
        gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx)
        assert bool(dx.isfinite().all()) and abs(loss.item() - ref.loss()[0]) <= ref.loss()[1]


def test_a_class_that_is_taken_out():
    """A bias of -inf: no part in lse, no gradient of its row of the table; a row of that class has an infinite loss and a finite gradient."""
    x, e, b, ids, _ = inputs(60, 40, 64, 0, F32, torch.int32, "common", 0, 0, True)
    ids[ids == 7] = 6
    b[7] = float("-inf")
    loss, lse = forward(x, e, b, ids, 60)
    others = torch.arange(40, device=dev()) != 7
    ids_without = torch.where(ids > 7, ids - 1, ids)
    loss2, lse2 = forward(x, e[others].contiguous(), b[others].contiguous(), ids_without, 60)
    assert torch.allclose(lse, lse2, rtol=1e-6, atol=0) and torch.allclose(loss, loss2, rtol=1e-6, atol=0)
    de, db = torch.empty_like(e), torch.empty_like(b)
    gsr.gsr_class_grad(x, e, ids, lse, dtable_out=de, bias=b, dbias_out=db)
    assert not de[7].any() and db[7] == 0 and bool(de.isfinite().all())
    ids[3] = 7
    loss, lse = forward(x, e, b, ids, 60)
    dx = torch.empty_like(x)
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b, dbias_out=db)
    assert loss.item() == float("inf") and bool(dx.isfinite().all()) and bool(de.isfinite().all()) and abs(db[7].item() + 1 / 60) <= 1e-7


@pytest.mark.parametrize("spread", ["classes", "rows", "columns", "learnt"])
def test_values_of_very_different_size(spread):
    """Classes of probabilities down to 1e-13, rows and columns of very different size, rows whose class is nearly certain.  Of the first two every row of
    every gradient is right to 1e-4 of its own largest value (its sums are of hundreds of terms, each right to 1e-5: logits of up to 30 are off by
    30 u and more)."""
    n, classes, d = 200, 300, 64
    rng = np.random.default_rng(11)
    x, e, b = rng.standard_normal((n, d)), rng.standard_normal((classes, d)) * 0.2, np.zeros(classes)
    if spread == "classes":
        b = -30.0 * rng.random(classes)
    elif spread == "rows":
        x *= np.exp(6.0 * rng.standard_normal((n, 1)).clip(-2, 0.3))
        e *= np.exp(4.0 * rng.standard_normal((classes, 1)).clip(-2, 0.3))
    elif spread == "columns":
        scale = np.exp(4.0 * rng.standard_normal(d))
        x, e = x * scale, e / scale
    ids = rng.integers(0, classes, n)
    if spread == "learnt":
        for i in range(n):
            x[i] += 15.0 * rng.random() * e[ids[i]] / (e[ids[i]] ** 2).sum()
    x, e, b, ids = put(x), put(e), put(b), torch.from_numpy(ids).to(dev())
    _, lse = forward(x, e, b, ids, n)
    ref = Reference(host(x), host(e), b.double().cpu().numpy(), ids.cpu().numpy(), F32)
    close(lse.double().cpu().numpy(), ref.lse, ref.lse_off)
    dx, de = torch.empty_like(x), torch.empty_like(e)
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b)
    want = ref.gradients(lse.double().cpu().numpy(), 1.0)
    for got, (exact, off) in ((host(dx), want["dx"]), (host(de), want["dtable"])):
        close(got, exact, off)
        if spread in ("classes", "rows"):
            assert (np.abs(got - exact) / np.abs(exact).max(1, keepdims=True)).max() <= 1e-4, spread


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bad_values_in_rows_without_a_class_have_no_part(dtype):
    x, e, b, ids, ref = inputs(100, 70, 64, 2, dtype, torch.int32, "common", 0, 0, True)
    ids[10:20] = -1
    ids[40] = 70
    loss, lse = forward(x, e, b, ids, 100)
    outs = lambda: (torch.empty_like(x), torch.empty_like(e), torch.empty_like(b))  # noqa: E731
    dx, de, db = outs()
    gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b, dbias_out=db)
    x[:, 10:20], x[:, 40] = float("nan"), float("inf")
    loss2, lse2 = forward(x, e, b, ids, 100)
    assert torch.equal(loss, loss2) and bool(lse2[10:20].isnan().all())
    dx2, de2, db2 = outs()
    gsr.gsr_class_grad(x, e, ids, lse2, dx_out=dx2, dtable_out=de2, bias=b, dbias_out=db2)
    assert torch.equal(dx, dx2) and torch.equal(de, de2) and torch.equal(db, db2)
    assert bool((dx[:, 10:20] == 0).all()) and bool((dx[:, 40] == 0).all())


def test_a_bad_row_with_a_class_shows_in_the_loss_and_its_own_lse_alone():
    x, e, b, ids, _ = inputs(100, 70, 64, 0, F32, torch.int32, "common", 0, 0, False)
    _, lse = forward(x, e, b, ids, 100)
    x[33, 5] = float("nan")
    loss, lse2 = forward(x, e, b, ids, 100)
    others = torch.arange(100, device=dev()) != 33
    assert bool(loss.isnan().all()) and bool(lse2[33].isnan()) and torch.equal(lse[others], lse2[others])


def test_ids_beyond_32_bits_are_no_classes():
    ids = torch.tensor([2 ** 32 + 1, 1, -2 ** 32, -2 ** 63, 2 ** 63 - 1, 0], device=dev())
    x, e = torch.randn((6, 16), device=dev()), torch.randn((4, 16), device=dev())
    loss, lse = forward(x, e, None, ids, 6)
    ref = Reference(host(x), host(e), np.zeros(4), ids.cpu().numpy(), F32)
    assert ref.count == 2 and abs(loss.item() - ref.loss()[0]) <= ref.loss()[1]


def test_nothing_to_learn_from():
    """No row, and no row with a class: loss 0, gradients 0."""
    e, b = torch.randn((40, 24), device=dev()), torch.randn(40, device=dev())
    for n in (0, 9):
        x, ids = torch.randn((n, 24), device=dev()), torch.full((n,), -1, device=dev())
        loss, lse = forward(x, e, b, ids, n)
        dx, de, db = torch.full_like(x, GUARD), torch.full_like(e, GUARD), torch.full_like(b, GUARD)
        gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b, dbias_out=db)
        assert loss.item() == 0.0 and not dx.any() and not de.any() and not db.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_and_replayed(dtype):
    n, classes, d = 700, 500, 128
    x, e, b, ids, _ = inputs(n, classes, d, 2, dtype, torch.int32, "mixed", 0, 0, True)
    ws = torch.empty(max(gsr.gsr_class_loss_workspace(x, classes), gsr.gsr_class_grad_workspace(x, classes)), dtype=torch.uint8, device=dev())

    def buffers():
        return dict(loss=torch.empty(1, device=dev()), lse=torch.empty(n, device=dev()), dx=torch.empty_like(x), de=torch.empty_like(e), db=torch.empty_like(b))

    def step(o, workspace=None):
        gsr.gsr_class_loss(x, e, ids, o["loss"], o["lse"], bias=b, workspace=workspace)
        gsr.gsr_class_grad(x, e, ids, o["lse"], dx_out=o["dx"], dtable_out=o["de"], bias=b, dbias_out=o["db"], workspace=workspace)

    got = buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(got, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got, ws)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        ids.copy_(torch.randint(-5, classes, (n,), device=dev(), dtype=torch.int32))
        ids[ids == classes // 2] = 0
        want = buffers()
        step(want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_calls_side_by_side_and_again_give_the_same_bits():
    n, classes, d = 5_000, 3_000, 256
    x, e, b, ids, _ = inputs(n, classes, d, 0, BF16, torch.int32, "common", 0, 0, True)

    def run():
        loss, lse = forward(x, e, b, ids, n)
        dx, de, db = torch.empty_like(x), torch.empty_like(e), torch.empty_like(b)
        gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b, dbias_out=db)
        return loss, lse, dx, de, db
    want = run()
    torch.cuda.synchronize()
    got = []
    for s in [torch.cuda.Stream() for _ in range(3)]:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(run())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_row_strides_that_lead_beyond_2_to_the_32_values():
    n, classes, d, stride = 35, 34, 64, 2 ** 27
    x, e, b, ids, _ = inputs(n, classes, d, 0, BF16, torch.int32, "mixed", 0, 0, True)
    memory = torch.empty(n * stride, dtype=BF16, device=dev())
    wide_x, wide_dx, wide_e, wide_de = (memory.as_strided((n if k < 2 else classes, d), (stride, 1), k * d) for k in range(4))
    wide_x.copy_(x)
    wide_e.copy_(e)

    def run(x, e, dx, de):
        loss, lse = forward(x, e, b, ids, n)
        gsr.gsr_class_grad(x, e, ids, lse, dx_out=dx, dtable_out=de, bias=b)
        return loss, lse, dx, de
    for got, want in zip(run(wide_x, wide_e, wide_dx, wide_de), run(x, e, torch.empty_like(x), torch.empty_like(e))):
        assert torch.equal(got, want)
