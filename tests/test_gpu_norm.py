"""Group norm over a batch of graphs, its gradient, and checkpoints in 8 bits, against the definitions in 64 bits.

u = 2^-24.  Forward: mean and rstd are rounded once; (x - m) r gamma + beta takes four more roundings, each of a value of at most
a = |gamma| r (|x| + |m|) + |beta|: 8 u a in all.  silu has a slope below 1.1 and, with exp(-z) off by (2 |z| + 4) u of itself and two more roundings in
the quotient, its own error is below (|z| (2 |z| + 6) / 4 + 2 |z|) u.  A 16-bit plane adds half a step, 2^-8 of the value.
Backward: a sum of up to 1,024 rows in 32 bits is off by 1,024 u times the sum of absolute values, every term by 16 u (silu: as above)."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from test_gpu_embed import BF16, F32, GUARD, dev, plane, rows_of, untouched

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ACTS = {"none": gsr.GSR_ACT_NONE, "relu": gsr.GSR_ACT_RELU, "silu": gsr.GSR_ACT_SILU}
EPS = 1e-5


def step_of(dtype):
    return 0.0 if dtype == F32 else 2.0 ** -8


def activation(z, act):
    return np.maximum(z, 0.0) if act == "relu" else z / (1.0 + np.exp(-z)) if act == "silu" else z


def slope(z, act):
    if act == "none":
        return np.ones_like(z)
    if act == "relu":
        return (z > 0.0).astype(np.float64)
    s = 1.0 / (1.0 + np.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def silu_error(z, act):
    z = np.abs(z)
    return (z * (2 * z + 6) / 4 + 2 * z) if act == "silu" else np.zeros_like(z)


class Reference:
    """Everything in float64 for rows x [n, d]; rows of no graph are NaN in what it returns."""

    def __init__(self, x, ptr, groups, gamma, beta, act, mean=None, rstd=None):
        self.x, self.ptr, self.groups, self.act = x, ptr, groups, act
        n, d = x.shape
        self.gamma = np.ones(d) if gamma is None else gamma
        self.beta = np.zeros(d) if beta is None else beta
        self.width = d // groups
        self.mean, self.rstd = mean, rstd
        if mean is None:
            self.mean, self.rstd = np.zeros((len(ptr) - 1, groups)), np.full((len(ptr) - 1, groups), 1.0 / np.sqrt(EPS))
            for s, a, b in self.spans():
                v = x[a:b].reshape(b - a, groups, self.width)
                self.mean[s] = v.mean((0, 2))
                self.rstd[s] = 1.0 / np.sqrt(((v - self.mean[s][:, None]) ** 2).mean((0, 2)) + EPS)

    def spans(self):
        return [(s, a, b) for s, (a, b) in enumerate(zip(self.ptr, self.ptr[1:])) if b > a]

    def of_rows(self, per_graph):
        out = np.full((len(self.x), self.groups * self.width), np.nan)
        for s, a, b in self.spans():
            out[a:b] = np.repeat(per_graph[s], self.width)
        return out

    def forward(self):
        """(y, bound of the error of a float32 y)."""
        m, r = self.of_rows(self.mean), self.of_rows(self.rstd)
        z = (self.x - m) * r * self.gamma + self.beta
        a = np.abs(self.gamma) * r * (np.abs(self.x) + np.abs(m)) + np.abs(self.beta)
        return activation(z, self.act), U * (1.1 * 8 * a + silu_error(z, self.act))

    def loss(self, dy):
        y = self.forward()[0]
        return np.nansum(y * dy)

    def backward(self, dy):
        """dx, dgamma, dbeta and the bounds of their errors in float32."""
        m, r = self.of_rows(self.mean), self.of_rows(self.rstd)
        known = ~np.isnan(m)
        xh = (self.x - m) * r
        z = xh * self.gamma + self.beta
        dz = dy * slope(z, self.act)
        a = r * (np.abs(self.x) + np.abs(m))                                    # roundings of xh are of this size
        # silu'' is below 0.6; its computed slope is off by the error of the logistic, below (2 |z| + 6) u, times 1 + 2 |z|
        off = np.abs(dy) * (16 + (0.6 * 8 * (a * np.abs(self.gamma) + np.abs(self.beta)) + (2 * np.abs(z) + 6) * (1 + 2 * np.abs(z))) * (self.act == "silu")) * U
        rows = min(len(self.x), 1024)
        sums = lambda v: np.where(known, v, 0.0).sum(0)                         # noqa: E731
        dx, dx_off = np.full_like(self.x, np.nan), np.full_like(self.x, np.nan)
        h, h_off = self.gamma * dz, np.abs(self.gamma) * (off + 2 * U * np.abs(dz))
        for s, p, q in self.spans():
            g = lambda v: v[p:q].reshape(q - p, self.groups, self.width)        # noqa: E731
            mean = lambda v: v.mean((0, 2))[:, None]                            # noqa: E731
            m1, m2 = mean(g(h)), mean(g(h * xh))
            m1_off = mean(g(h_off)) + (rows + 4) * U * mean(np.abs(g(h)))
            m2_off = mean(g(h_off * np.abs(xh) + 4 * U * np.abs(h) * a)) + (rows + 4) * U * mean(np.abs(g(h * xh)))
            rr = g(r)
            dx[p:q] = (rr * (g(h) - m1 - g(xh) * m2)).reshape(q - p, -1)
            size = np.abs(g(h)) + np.abs(m1) + np.abs(g(xh) * m2)
            dx_off[p:q] = (rr * (g(h_off) + m1_off + np.abs(g(xh)) * m2_off + 4 * U * g(a) * np.abs(m2) + 8 * U * size)).reshape(q - p, -1)
        return dict(dx=dx, dgamma=sums(dz * xh), dbeta=sums(dz)), dict(
            dx=dx_off, dgamma=sums(off * np.abs(xh) + 4 * U * np.abs(dz) * a) + (rows + 4) * U * sums(np.abs(dz * xh)),
            dbeta=sums(off) + (rows + 4) * U * sums(np.abs(dz)))


def borders(kind, n, rng):
    """First rows of graphs."""
    if kind == "one":
        return None
    if kind == "rows":
        return np.arange(n + 1)
    if kind == "padded":                            # rows before the first and behind the last
        return np.sort(np.concatenate([[n // 7, n - n // 5], rng.integers(n // 7, n - n // 5 + 1, 5)]))
    if kind == "empty":
        return np.array([0, 0, 0, n // 3, n // 3, n, n, n])
    if kind == "none":
        return np.array([n // 2])
    if kind == "uneven":                            # two large graphs among small ones
        sizes = [n // 500] * 13 + [n * 2 // 5] + [n // 250] * 14 + [n * 2 // 5] + [n // 500] * 10
        return np.concatenate([[0], np.cumsum(sizes), [n]])
    assert kind == "many"
    return np.sort(np.concatenate([[0, n], rng.integers(0, n + 1, max(1, n // 6))]))


def arrays(n, d, rng):
    x = rng.standard_normal((n, d)) * np.exp(0.5 * rng.standard_normal((n, 1))) + rng.standard_normal(d)
    return x, 1.0 + 0.3 * rng.standard_normal(d), 0.3 * rng.standard_normal(d)


def put(a, dtype=F32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(dev())


def host(t):
    return rows_of(t).double().cpu().numpy()


def close(got, want, off, dtype=F32):
    """Everywhere where `want` is a number."""
    known = ~np.isnan(want)
    allowed = off + (np.abs(want) + off) * step_of(dtype) + 2.0 ** -149
    worst = (np.abs(got - want) - allowed)[known]
    assert worst.size == 0 or worst.max() <= 0.0, (worst.max(), np.abs(got - want)[known].max())


CASES = [
    # n, d, c, groups, dtype, act, graphs, pad, offset, affine
    (1, 1, 0, 1, F32, "none", "one", 0, 0, True),
    (1, 64, 2, 2, F32, "relu", "one", 0, 0, True),
    (1, 64, 0, 8, BF16, "silu", "one", 0, 0, False),
    (2, 3, 0, 1, F32, "silu", "rows", 2, 1, True),
    (3, 40, 0, 5, BF16, "relu", "rows", 0, 0, True),
    (100, 5, 0, 5, F32, "none", "many", 0, 3, True),
    (101, 64, 2, 2, F32, "relu", "one", 0, 0, True),
    (257, 64, 2, 1, F32, "silu", "padded", 0, 0, True),
    (1000, 96, 3, 2, F32, "silu", "many", 0, 0, True),            # a group lies across planes
    (1001, 77, 0, 7, F32, "relu", "many", 1, 1, True),
    (1001, 77, 0, 11, BF16, "silu", "empty", 3, 1, True),
    (999, 256, 8, 32, BF16, "relu", "many", 0, 0, True),
    (999, 256, 4, 4, F32, "none", "padded", 4, 2, False),
    (513, 384, 2, 6, F32, "silu", "empty", 0, 0, True),
    (300, 514, 0, 2, BF16, "none", "many", 0, 0, True),
    (64, 1028, 0, 1, F32, "relu", "many", 0, 0, True),
    (33, 2056, 2, 4, BF16, "silu", "padded", 8, 8, True),
    (5, 131_072, 0, 64, F32, "silu", "empty", 0, 0, True),
    (70, 6, 6, 6, F32, "relu", "many", 0, 0, True),
    (20_011, 64, 0, 4, F32, "silu", "many", 0, 0, True),
    (40_000, 128, 2, 2, BF16, "relu", "padded", 0, 0, True),
    (9_000, 33, 0, 3, BF16, "silu", "one", 0, 0, True),
    # widths that are no whole number of pieces, one group: the last piece of a row overlaps the one before
    (1001, 77, 0, 1, F32, "silu", "many", 1, 1, True),
    (1003, 385, 0, 1, BF16, "relu", "padded", 0, 0, True),
    (517, 130, 2, 1, BF16, "silu", "many", 0, 0, True),
    (517, 134, 2, 1, F32, "none", "empty", 3, 2, True),
    (90, 257, 0, 1, F32, "relu", "rows", 0, 0, False),
    (70, 9, 0, 1, BF16, "silu", "many", 0, 1, True),
    (41, 1031, 0, 1, BF16, "none", "padded", 0, 0, True),
    # groups that are no whole number of pieces: they begin and end inside one
    (703, 99, 3, 9, F32, "silu", "many", 0, 0, True),
    (703, 150, 2, 6, BF16, "relu", "padded", 0, 0, True),
    (301, 1020, 0, 12, F32, "silu", "many", 0, 0, True),
    (203, 2055, 0, 15, BF16, "silu", "many", 1, 1, True),
    (500, 136, 0, 8, F32, "relu", "one", 0, 0, True),
    (500, 136, 0, 8, BF16, "relu", "many", 0, 0, False),
    (400, 90, 2, 3, F32, "none", "empty", 0, 0, True),
    (400, 102, 2, 3, BF16, "silu", "padded", 2, 0, True),
    (61, 5000, 0, 8, F32, "relu", "rows", 0, 0, True),
    (5_000, 64, 0, 1, F32, "silu", "uneven", 0, 0, True),
    (5_003, 96, 2, 4, BF16, "relu", "uneven", 0, 0, True),
    (6_001, 99, 0, 3, F32, "none", "uneven", 1, 0, True),
    (50, 48, 0, 3, F32, "silu", "none", 0, 0, True),
    (0, 48, 0, 3, F32, "silu", "none", 0, 0, True),
]


def case_inputs(n, d, c, groups, dtype, graphs, pad, offset, affine):
    rng = np.random.default_rng(n + d)
    x, gamma, beta = arrays(n, d, rng)
    gamma, beta = (gamma.astype(np.float32).astype(np.float64), beta.astype(np.float32).astype(np.float64)) if affine else (None, None)
    buffer, px = plane(n, d, c, dtype, torch.from_numpy(x), pad, offset)
    ptr = borders(graphs, n, rng)
    index = torch.int32 if n % 2 else torch.int64
    return rng, host(px), px, gamma, beta, (np.array([0, n]) if ptr is None else ptr), (None if ptr is None else put(ptr, index))


def stats(ptr, groups):
    return (torch.full((len(ptr) - 1, groups), GUARD, device=dev()) for _ in range(2))


@pytest.mark.parametrize("n,d,c,groups,dtype,act,graphs,pad,offset,affine", CASES)
def test_forward(n, d, c, groups, dtype, act, graphs, pad, offset, affine):
    rng, x, px, gamma, beta, ptr, dptr = case_inputs(n, d, c, groups, dtype, graphs, pad, offset, affine)
    buffer, y = plane(n, d, c, dtype, None, pad, offset)
    mean, rstd = stats(ptr, groups)
    gsr.gsr_group_norm(px, y, mean, rstd, gamma=put(gamma), beta=put(beta), eps=EPS, act=ACTS[act], graph_ptr=dptr)
    ref = Reference(x, ptr, groups, gamma, beta, act)
    close(mean.double().cpu().numpy(), ref.mean, 2 * U * np.abs(ref.mean))
    close(rstd.double().cpu().numpy(), ref.rstd, 2 * U * ref.rstd)
    want, off = ref.forward()
    close(host(y), want, off, dtype)
    assert np.all(host(y)[np.isnan(want)] == GUARD) and untouched(buffer, y)


@pytest.mark.parametrize("n,d,c,groups,dtype,act,graphs,pad,offset,affine", CASES)
def test_gradient(n, d, c, groups, dtype, act, graphs, pad, offset, affine):
    rng, x, px, gamma, beta, ptr, dptr = case_inputs(n, d, c, groups, dtype, graphs, pad, offset, affine)
    _, dy = plane(n, d, c, dtype, torch.from_numpy(rng.standard_normal((n, d))), pad, offset)
    buffer, dx = plane(n, d, c, dtype, None, pad, offset)
    exact = Reference(x, ptr, groups, gamma, beta, act)
    mean, rstd = put(exact.mean), put(exact.rstd)
    dgamma, dbeta = (torch.full((d,), GUARD, device=dev()) for _ in range(2))
    gsr.gsr_group_norm_grad(dy, mean, rstd, dx, x=px, gamma=put(gamma), beta=put(beta), act=ACTS[act], graph_ptr=dptr, dgamma_out=dgamma, dbeta_out=dbeta)
    ref = Reference(x, ptr, groups, gamma, beta, act, mean.double().cpu().numpy(), rstd.double().cpu().numpy())
    want, off = ref.backward(host(dy))
    close(host(dx), want["dx"], off["dx"], dtype)
    assert np.all(host(dx)[np.isnan(want["dx"])] == GUARD) and untouched(buffer, dx)
    close(dgamma.double().cpu().numpy(), want["dgamma"], off["dgamma"])
    close(dbeta.double().cpu().numpy(), want["dbeta"], off["dbeta"])


@pytest.mark.parametrize("act", ["none", "silu", "relu"])
def test_gradient_against_differences(act):
    """The kernel's gradients along random directions against differences of the loss sum(y dy) in 64 bits."""
    n, d, groups = 60, 24, 3
    rng = np.random.default_rng(5)
    x, gamma, beta = arrays(n, d, rng)
    x, gamma, beta, dy = (v.astype(np.float32).astype(np.float64) for v in (x, gamma, beta, rng.standard_normal((n, d))))
    ptr = np.array([0, 7, 7, 41, 60])
    mean, rstd = stats(ptr, groups)
    y, dx, dgamma, dbeta = torch.empty((n, d), device=dev()), torch.empty((n, d), device=dev()), torch.empty(d, device=dev()), torch.empty(d, device=dev())
    args = dict(gamma=put(gamma), beta=put(beta), act=ACTS[act], graph_ptr=put(ptr, torch.int64))
    gsr.gsr_group_norm(put(x), y, mean, rstd, eps=EPS, **args)
    gsr.gsr_group_norm_grad(put(dy), mean, rstd, dx, x=put(x), dgamma_out=dgamma, dbeta_out=dbeta, **args)
    h = 1e-6
    for i, (got, at) in enumerate(((dx, x), (dgamma, gamma), (dbeta, beta))):
        v = rng.standard_normal(at.shape)
        def loss(t, i=i, v=v):
            moved = [x, gamma, beta]
            moved[i] = moved[i] + t * v
            return Reference(moved[0], ptr, groups, moved[1], moved[2], act).loss(dy)
        slope_at = (loss(h) - loss(-h)) / (2 * h)
        along = float((got.double().cpu().numpy() * v).sum())
        # differences: h^2 times third derivatives, below 1e-9; cancellation 2^-53 * 1e3 / h; the kernel: 1e-6 of every term
        assert abs(along - slope_at) <= 1e-5 * np.abs(got.double().cpu().numpy() * v).sum() + 1e-6, (act, i)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,c,groups", [(701, 128, 2, 4), (701, 77, 0, 1), (300, 257, 0, 1), (300, 77, 0, 7), (300, 136, 0, 8), (200, 150, 2, 6)])
def test_in_place(dtype, n, d, c, groups):
    rng, x, px, gamma, beta, ptr, dptr = case_inputs(n, d, c, groups, dtype, "padded", 0, 0, True)
    args = dict(gamma=put(gamma), beta=put(beta), act=gsr.GSR_ACT_SILU, graph_ptr=dptr)
    mean, rstd = stats(ptr, groups)
    y = torch.full_like(px, 0.0)
    y.copy_(px)                                       # rows of no graph keep their values in place
    gsr.gsr_group_norm(px, y, mean, rstd, **args)
    before, mean2, rstd2 = px.clone(), mean.clone(), rstd.clone()
    gsr.gsr_group_norm(px, px, mean2, rstd2, **args)
    # (odd widths are taken in other pieces in place: sums of statistics in 64 bits, joined in another order, are rounded to the same or the next float)
    assert torch.allclose(mean, mean2, rtol=2 * U, atol=0) and torch.allclose(rstd, rstd2, rtol=2 * U, atol=0)
    if torch.equal(mean, mean2) and torch.equal(rstd, rstd2):
        assert torch.equal(px, y)
    dy = torch.randn(px.shape, device=dev()).to(dtype)
    dx, given = dy.clone(), host(dy)
    gsr.gsr_group_norm_grad(dy, mean, rstd, dx, x=before, **args)
    gsr.gsr_group_norm_grad(dy, mean, rstd, dy, x=before, **args)
    ref = Reference(x, ptr, groups, gamma, beta, "silu", mean.double().cpu().numpy(), rstd.double().cpu().numpy())
    if d % groups == 0 and d // groups % 8 == 0 and d // max(c, 1) % 8 == 0:
        assert torch.equal(dx, dy)
    want, off = ref.backward(given)
    close(host(dy), np.where(np.isnan(want["dx"]), np.nan, want["dx"]), off["dx"], dtype)
    assert torch.equal(rows_of(dy)[:ptr[0]], torch.from_numpy(given[:ptr[0]]).to(dtype).to(dev()))


@pytest.mark.parametrize("n,ptr", [(5_000, None), (60_000, None), (9_000, [0, 4_000, 4_000, 9_000])])
def test_a_constant_group_and_far_means(n, ptr):
    """Variance 0 gives rstd = 1 / sqrt(eps) and y = beta.  A mean of 10,000 or a million standard deviations leaves rstd right: values are summed from the first one
    on, a few standard deviations from all, so that 64 bits lose below 2^13 additions * 2^-53 * 100 of the variance, less than half a float's step."""
    graphs = [0, n] if ptr is None else ptr
    dptr = None if ptr is None else torch.tensor(ptr, device=dev())
    x = torch.full((n, 8), 3.25, device=dev())
    y, (mean, rstd) = torch.empty_like(x), stats(graphs, 2)
    beta = torch.arange(8.0, device=dev())
    gsr.gsr_group_norm(x, y, mean, rstd, beta=beta, graph_ptr=dptr)
    empty = torch.tensor([a == b for a, b in zip(graphs, graphs[1:])], device=dev())[:, None].expand(-1, 2)
    assert torch.equal(mean, torch.where(empty, 0.0, 3.25).float()) and torch.equal(y, beta.expand(n, 8))
    assert torch.equal(rstd, torch.full_like(rstd, 1.0 / np.sqrt(np.float64(np.float32(1e-5)))))
    for off in (1e4, 1e6):
        far = torch.randn((n, 8), generator=torch.Generator(device="cuda").manual_seed(1), device=dev()) + off
        gsr.gsr_group_norm(far, torch.empty_like(far), mean, rstd, graph_ptr=dptr)
        ref = Reference(far.double().cpu().numpy(), np.array(graphs), 2, None, None, "none")
        close(mean.double().cpu().numpy(), ref.mean, 2 * U * np.abs(ref.mean))
        close(rstd.double().cpu().numpy(), ref.rstd, 2 * U * ref.rstd)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_bad_value_stays_in_its_graph_and_group(bad):
    x = torch.randn((90, 64), device=dev())
    ptr = torch.tensor([0, 30, 60, 90], device=dev())
    y, y2, (mean, rstd) = torch.empty_like(x), torch.empty_like(x), stats([0, 30, 60, 90], 4)
    gsr.gsr_group_norm(x, y, mean, rstd, graph_ptr=ptr)
    x[45, 20] = bad
    gsr.gsr_group_norm(x, y2, mean, rstd, graph_ptr=ptr)
    hit = torch.zeros((90, 64), dtype=torch.bool, device=dev())
    hit[30:60, 16:32] = True
    assert bool(y2[hit].isnan().all()) and torch.equal(y2[~hit], y[~hit])


def test_bad_values_in_rows_of_no_graph_have_no_part():
    x = torch.randn((90, 64), device=dev())
    x[:10], x[80:] = float("nan"), float("inf")
    ptr = torch.tensor([10, 50, 80], dtype=torch.int32, device=dev())
    y, (mean, rstd) = torch.full_like(x, GUARD), stats([10, 50, 80], 4)
    gsr.gsr_group_norm(x, y, mean, rstd, graph_ptr=ptr, act=gsr.GSR_ACT_RELU)
    assert bool(y[10:80].isfinite().all()) and bool((y[:10] == GUARD).all()) and bool((y[80:] == GUARD).all())
    dx, dgamma = torch.full_like(x, GUARD), torch.empty(64, device=dev())
    gsr.gsr_group_norm_grad(x, mean, rstd, dx, x=x, graph_ptr=ptr, act=gsr.GSR_ACT_SILU, dgamma_out=dgamma)
    assert bool(dx[10:80].isfinite().all()) and bool((dx[:10] == GUARD).all()) and bool((dx[80:] == GUARD).all()) and bool(dgamma.isfinite().all())


def test_offsets_beyond_the_plane_count_as_its_border():
    x = torch.randn((50, 32), device=dev())
    want, got, (mean, rstd) = torch.full_like(x, GUARD), torch.full_like(x, GUARD), stats([0, 20, 50], 2)
    mean2, rstd2 = mean.clone(), rstd.clone()
    gsr.gsr_group_norm(x, want, mean, rstd, graph_ptr=torch.tensor([0, 20, 50], device=dev()))
    gsr.gsr_group_norm(x, got, mean2, rstd2, graph_ptr=torch.tensor([-7, 20, 2 ** 40], device=dev()))
    assert torch.equal(want, got) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)


# ---- checkpoints ------------------------------------------------------------------------------------------------
LARGEST = np.nextafter(np.finfo(np.float32).max / np.float32(127.0), np.float32(0.0))          # the quotient itself, times 127, is infinite


def codes_ref(x, c):
    """codes and scales of rows x (float32 or wider values) in max(c, 1) groups, group by group: exact products in 64 bits."""
    n, d = x.shape
    dg = d // max(c, 1)
    codes, scales = np.zeros((n, d), dtype=np.int8), []
    for i in range(max(c, 1)):
        for a in range(0, dg, 64):
            lo, hi = i * dg + a, i * dg + min(dg, a + 64)
            part = x[:, lo:hi].astype(np.float64)
            fine = np.isfinite(part).all(1)
            part = np.where(fine[:, None], part, 0.0)
            top = np.maximum(np.abs(part).max(1), 127.0 * 2.0 ** -126)
            codes[:, lo:hi] = np.rint(127.0 * part / top[:, None]).astype(np.int8)       # 127 x is exact, the quotient rounded to 53 bits
            scale = np.minimum(top.astype(np.float32) / np.float32(127.0), LARGEST)
            scales.append(np.where(fine, scale, np.float32(np.nan)))
    by_group = lambda v: np.ascontiguousarray(v.reshape(n, max(c, 1), v.shape[1] // max(c, 1)).transpose(1, 0, 2))         # noqa: E731
    return by_group(codes), by_group(np.stack(scales, 1))


def decoded(codes, scales, c):
    """The rows [n, d] that codes and scales in the order of a plane of max(c, 1) groups stand for, in float32."""
    (n, d), c = codes.shape, max(c, 1)
    q, s = codes.view(c, n, d // c), scales.view(c, n, scales.shape[1] // c)
    blocks = torch.arange(q.shape[2], device=dev()) // 64
    return (q.float() * s[:, :, blocks]).permute(1, 0, 2).reshape(n, d)


def save(x, n, d, c):
    codes = torch.full((n, d), 77, dtype=torch.int8, device=dev())
    scales = torch.full((n, gsr.gsr_checkpoint_blocks(d, max(c, 1))), GUARD, device=dev())
    gsr.gsr_checkpoint_save(x, codes, scales)
    return codes, scales


@pytest.mark.parametrize("n,d,c,dtype,pad,offset", [
    (1, 1, 0, F32, 0, 0), (1, 3, 0, BF16, 2, 1), (7, 64, 2, F32, 0, 0), (7, 64, 0, BF16, 0, 0), (100, 77, 0, F32, 1, 3), (101, 257, 0, BF16, 1, 1),
    (1001, 256, 4, F32, 0, 0), (1001, 256, 8, BF16, 0, 0), (500, 384, 2, F32, 0, 0), (333, 80, 2, F32, 4, 2), (333, 80, 2, BF16, 0, 0),
    (64, 24, 6, F32, 0, 0), (9, 2052, 0, F32, 0, 0), (200, 130, 2, F32, 0, 0), (200, 134, 2, BF16, 0, 0), (200, 126, 2, BF16, 3, 1), (77, 191, 0, BF16, 0, 1),
    (77, 385, 0, BF16, 0, 0), (50, 9, 0, BF16, 0, 0), (50, 5, 0, F32, 1, 0), (41, 1031, 0, F32, 0, 0), (1000, 515, 0, BF16, 0, 0), (60, 198, 3, F32, 0, 0), (30_000, 64, 0, BF16, 8, 8), (3, 131_072, 0, F32, 0, 0), (0, 64, 0, F32, 0, 0)])
def test_checkpoint(n, d, c, dtype, pad, offset):
    rng = np.random.default_rng(n + d)
    values = rng.standard_normal((n, d)) * np.exp(3.0 * rng.standard_normal((n, 1)))
    _, x = plane(n, d, c, dtype, torch.from_numpy(values), pad, offset)
    codes, scales = save(x, n, d, c)
    want, want_scales = codes_ref(rows_of(x).float().cpu().numpy(), c)
    assert np.array_equal(codes.cpu().numpy().ravel(), want.ravel()) and np.array_equal(scales.cpu().numpy().ravel(), want_scales.ravel())
    buffer, back = plane(n, d, c, dtype, None, pad, offset)
    gsr.gsr_checkpoint_load(codes, scales, back)
    assert torch.equal(rows_of(back), decoded(codes, scales, c).to(dtype)) and untouched(buffer, back)


def test_checkpoint_at_the_borders_between_codes():
    """Halves of the largest value are ties (63.5), and so are multiples of it by odd numbers of 254ths where these are exact; their neighbours are not."""
    rows = []
    for top in (1.0, 254.0, 127.0 * 2.0 ** -30, 3.0, 1.9999998807907104, 2.0 ** 100, 2.0 ** -100):
        k = np.arange(1, 254, 4, dtype=np.float64)[:62]
        near = (top * k / 254.0).astype(np.float32)
        for v in (near, np.nextafter(near, np.float32(np.inf)), np.nextafter(near, np.float32(0))):
            rows.append(np.concatenate([[top, top / 2], v * np.where(np.arange(62) % 2, -1, 1)]))
    x = np.array(rows, dtype=np.float32)
    codes, scales = save(put(x), *x.shape, 0)
    want, want_scales = codes_ref(x, 0)
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scales.cpu().numpy(), want_scales[0])
    assert np.all(want[0, :, 1] == 64)


def test_checkpoint_of_extreme_values():
    """Zeros, the smallest and the largest floats, infinities and NaN: the last two take their block with them and nothing else."""
    x = torch.zeros((8, 128), device=dev())
    x[1, 5] = 2.0 ** -149
    x[2, 64:] = -(2.0 ** -130)
    x[3] = torch.finfo(F32).max
    x[4, 3], x[4, 64:] = float("inf"), 1.0
    x[5, 70], x[5, :64] = float("nan"), -2.0
    x[6, 0], x[6, 1] = float("-inf"), float("nan")
    x[7] = torch.linspace(-1e30, 1e-30, 128)
    codes, scales = save(x, 8, 128, 0)
    want, want_scales = codes_ref(x.cpu().numpy(), 0)
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scales.cpu().numpy(), want_scales[0], equal_nan=True)
    back = torch.empty_like(x)
    gsr.gsr_checkpoint_load(codes, scales, back)
    assert bool(back[4, :64].isnan().all()) and bool((back[4, 64:] - 1.0).abs().max() <= 2.0 ** -23) and bool(back[5, 64:].isnan().all())
    assert bool((back[5, :64] + 2.0).abs().max() <= 2.0 ** -22) and bool(back[6, :64].isnan().all()) and bool((back[6, 64:] == 0).all())
    assert bool((back[0] == 0).all()) and bool(back[3].isfinite().all()) and bool((back[3] / torch.finfo(F32).max - 1.0).abs().max() <= 2.0 ** -22)


@pytest.mark.parametrize("n,d,c,groups,dtype,graphs", [(1001, 256, 4, 4, F32, "padded"), (777, 77, 0, 7, BF16, "many"), (64, 96, 3, 6, BF16, "one"),
                                                       (333, 40, 0, 2, F32, "empty"), (333, 77, 0, 1, F32, "many"), (201, 130, 2, 1, BF16, "padded"), (333, 150, 2, 6, BF16, "many"), (333, 99, 3, 9, F32, "padded"),
                                                       (99, 385, 0, 1, BF16, "one")])
def test_norm_writes_the_checkpoint_and_its_gradient_reads_it(n, d, c, groups, dtype, graphs):
    rng, x, px, gamma, beta, ptr, dptr = case_inputs(n, d, c, groups, dtype, graphs, 0, 0, True)
    args = dict(gamma=put(gamma), beta=put(beta), act=gsr.GSR_ACT_SILU, graph_ptr=dptr)
    mean, rstd = stats(ptr, groups)
    y, y8 = torch.full_like(px, GUARD), torch.full_like(px, GUARD)
    gsr.gsr_group_norm(px, y, mean, rstd, **args)
    codes, scales = torch.full((n, d), 77, dtype=torch.int8, device=dev()), torch.full((n, gsr.gsr_checkpoint_blocks(d, max(c, 1))), GUARD, device=dev())
    mean8, rstd8 = mean.clone(), rstd.clone()
    gsr.gsr_group_norm(px, y8, mean8, rstd8, codes_out=codes, scales_out=scales, **args)
    assert torch.equal(y, y8) and torch.equal(mean, mean8) and torch.equal(rstd, rstd8)
    whole_codes, whole_scales = save(px, n, d, c)
    a, b = int(ptr[0]), int(ptr[-1])
    by_rows = lambda v: v.view(max(c, 1), n, -1)                                                       # noqa: E731
    for got, whole, guard in ((by_rows(codes), by_rows(whole_codes), 77), (by_rows(scales), by_rows(whole_scales), GUARD)):
        assert torch.equal(got[:, a:b], whole[:, a:b]) and bool((got[:, :a] == guard).all()) and bool((got[:, b:] == guard).all())
    # the gradient from the codes is that of the values they stand for
    _, dy = plane(n, d, c, dtype, torch.from_numpy(rng.standard_normal((n, d))))
    dx, dgamma, dbeta = torch.full_like(px, GUARD), torch.empty(d, device=dev()), torch.empty(d, device=dev())
    gsr.gsr_group_norm_grad(dy, mean, rstd, dx, codes=codes, scales=scales, dgamma_out=dgamma, dbeta_out=dbeta, **args)
    stands_for = decoded(whole_codes, whole_scales, c).double().cpu().numpy()
    ref = Reference(stands_for, ptr, groups, gamma, beta, "silu", mean.double().cpu().numpy(), rstd.double().cpu().numpy())
    want, off = ref.backward(host(dy))
    close(host(dx), want["dx"], off["dx"], dtype)
    close(dgamma.double().cpu().numpy(), want["dgamma"], off["dgamma"])
    close(dbeta.double().cpu().numpy(), want["dbeta"], off["dbeta"])


@pytest.mark.parametrize("n,d,groups,graphs", [(40_000, 16, 16, 30_000), (3_000, 2_048, 2_048, 600)])
def test_many_graphs_and_groups(n, d, groups, graphs):
    """More sums than workgroups are launched for, and groups of single columns."""
    rng = np.random.default_rng(n)
    x = rng.standard_normal((n, d)).astype(np.float32)
    ptr = np.sort(np.concatenate([[0, n], rng.integers(0, n + 1, graphs - 1)]))
    y, (mean, rstd) = torch.empty((n, d), device=dev()), stats(ptr, groups)
    gsr.gsr_group_norm(put(x), y, mean, rstd, eps=EPS, graph_ptr=put(ptr, torch.int64))
    graph = np.repeat(np.arange(graphs), np.diff(ptr))
    sums = lambda v: np.add.reduceat(np.concatenate([v, np.zeros((1, d))]), ptr[:-1], axis=0) * (np.diff(ptr) > 0)[:, None]     # noqa: E731
    count = np.maximum(np.diff(ptr), 1)[:, None]
    x = x.astype(np.float64)
    m = sums(x) / count
    r = 1.0 / np.sqrt(sums((x - m[graph]) ** 2) / count + EPS)
    close(mean.double().cpu().numpy(), m, 2 * U * np.abs(m) + 1e-15)
    close(rstd.double().cpu().numpy(), r, 2 * U * r + 1e-13 * r ** 3)
    assert torch.equal(y, (put(x) - mean[graph]) * rstd[graph]) or (y - (put(x) - mean[graph]) * rstd[graph]).abs().max() <= 4 * U * 320


def test_captured_and_replayed():
    """Both directions and a checkpoint in one graph, replayed on other inputs with eager work between."""
    n, d, groups = 3000, 128, 4
    rng, _, x, gamma, beta, ptr, dptr = case_inputs(n, d, 2, groups, F32, "padded", 0, 0, True)
    args = dict(gamma=put(gamma), beta=put(beta), act=gsr.GSR_ACT_RELU, graph_ptr=dptr)
    dy = torch.randn_like(x)
    ws = torch.empty(gsr.gsr_group_norm_workspace(x, groups, dptr), dtype=torch.uint8, device=dev())

    def buffers():
        mean, rstd = stats(ptr, groups)
        return dict(y=torch.full_like(x, GUARD), mean=mean, rstd=rstd, dx=torch.full_like(x, GUARD), dgamma=torch.empty(d, device=dev()),
                    codes=torch.zeros((n, d), dtype=torch.int8, device=dev()), scales=torch.zeros((n, 2), device=dev()))

    def step(o, workspace=None):
        gsr.gsr_group_norm(x, o["y"], o["mean"], o["rstd"], codes_out=o["codes"], scales_out=o["scales"], workspace=workspace, **args)
        gsr.gsr_group_norm_grad(dy, o["mean"], o["rstd"], o["dx"], codes=o["codes"], scales=o["scales"], dgamma_out=o["dgamma"], workspace=workspace, **args)

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
        x.copy_(torch.randn_like(x) + 0.5)
        dy.copy_(torch.randn_like(dy))
        want = buffers()
        step(want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_calls_side_by_side_and_again_give_the_same_bits():
    n, d, groups = 20_000, 256, 8
    x = torch.randn((n, d), device=dev())
    dy = torch.randn((n, d), device=dev())
    ptr = torch.tensor([0, 100, 9_000, n], device=dev())
    def run():
        y, (mean, rstd) = torch.empty_like(x), stats([0, 1, 2, 3], groups)
        dx, dgamma, dbeta = torch.empty_like(x), torch.empty(d, device=dev()), torch.empty(d, device=dev())
        gsr.gsr_group_norm(x, y, mean, rstd, act=gsr.GSR_ACT_SILU, graph_ptr=ptr)
        gsr.gsr_group_norm_grad(dy, mean, rstd, dx, x=x, act=gsr.GSR_ACT_SILU, graph_ptr=ptr, dgamma_out=dgamma, dbeta_out=dbeta)
        return y, mean, rstd, dx, dgamma, dbeta
    want = run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(run())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


@pytest.mark.parametrize("c", [0, 4])
def test_planes_of_more_than_2_to_the_32_values(c):
    """The last graph of a plane whose values, codes and their offsets pass 32 bits, against the same rows by themselves.

    Sums of other chunks: means of h and h xh are off by 1,024 u of the mean of absolute values (below 1) in each call, so dx by 2 * 1,024 u * (1 + |xh|) r, below
    2^-10 for |xh| < 7; and every 16-bit result by half a step in each, 2^-7 of the value for both."""
    n, d, last = 17_000_001, 256, 1_003
    torch.manual_seed(1)
    x = torch.empty((n, d) if not c else (c, n, d // c), dtype=BF16, device=dev()).normal_()
    blocks = gsr.gsr_checkpoint_blocks(d, max(1, c))
    y, codes, scales = torch.empty_like(x), torch.empty(x.shape, dtype=torch.int8, device=dev()), torch.empty((*x.shape[:-1], blocks // max(1, c)), device=dev())
    ptr = torch.tensor([0, n - last, n], device=dev())
    mean, rstd = stats([0, 1, 2], 8)
    gsr.gsr_group_norm(x, y, mean, rstd, graph_ptr=ptr, codes_out=codes, scales_out=scales)

    def end(t):
        return t[..., -last:, :].contiguous()
    x2 = end(x)
    y2, codes2, scales2 = torch.empty_like(x2), torch.empty(x2.shape, dtype=torch.int8, device=dev()), torch.empty((*x2.shape[:-1], blocks // max(1, c)), device=dev())
    mean2, rstd2 = stats([0, 1], 8)
    gsr.gsr_group_norm(x2, y2, mean2, rstd2, codes_out=codes2, scales_out=scales2)
    assert torch.equal(end(codes), codes2) and torch.equal(end(scales), scales2)
    assert torch.allclose(mean[1:], mean2, rtol=4 * U, atol=1e-12) and torch.allclose(rstd[1:], rstd2, rtol=4 * U)
    assert torch.allclose(end(y).float(), y2.float(), rtol=2.0 ** -7, atol=16 * U * 8)
    assert float(y[..., :1000, :].float().std()) > 0.9
    back, back2 = torch.empty_like(x2), torch.empty_like(x2)
    gsr.gsr_checkpoint_load(codes, scales, x)
    gsr.gsr_checkpoint_load(codes2, scales2, back2)
    back.copy_(end(x))
    assert torch.equal(back, back2)
    dy2 = end(y)
    dx2 = torch.empty_like(dy2)
    gsr.gsr_group_norm_grad(dy2, mean[1:].contiguous(), rstd[1:].contiguous(), dx2, codes=codes2, scales=scales2)
    gsr.gsr_group_norm_grad(y, mean, rstd, y, codes=codes, scales=scales, graph_ptr=ptr)
    assert torch.allclose(end(y).float(), dx2.float(), rtol=2.0 ** -7, atol=2.0 ** -10)
