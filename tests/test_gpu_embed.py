"""Embedding lookup and its gradient against the definitions in 64 bits.

Lookup rounds scale * E once, as torch's float32 product does, so outputs are compared bit for bit.  The gradient of whole numbers is
exact in float32 whatever the order of the sum, so it is too; of other numbers every addition is off by at most 2^-24 of a partial sum,
which no sum of absolute values exceeds.  A row takes at most 256 additions in its chunk, 32 on each of at most four levels above
(n < 2^31), 80 where a run is joined, and the scale one rounding: |error| <= 465 * 2^-24 scale sum |dx|."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
GUARD = -7.0


def dev():
    return torch.device("cuda:0")


def make_ids(kind, n, vocab, rng):
    """Tokens as int64 numpy: one of all, all different, a few common ones, with and without tokens outside the table."""
    if kind == "one":
        return np.full(n, vocab - 1)
    if kind == "distinct":
        return np.resize(rng.permutation(vocab), n)
    if kind == "common":
        return np.minimum((vocab + 1.0) ** rng.random(n) - 1, vocab - 1).astype(np.int64)
    if kind == "unknown":
        return np.where(np.arange(n) % 2 == 0, -1, vocab)
    assert kind == "mixed"
    ids = rng.integers(0, vocab, n)
    ids[rng.random(n) < 0.2] = -1
    ids[rng.random(n) < 0.1] = vocab
    return ids


def plane(n, d, c, dtype, values=None, pad=0, offset=0):
    """A plane [n, d] (c = 0) or [c, n, d / c] whose rows lie `pad` elements apart, in a buffer of GUARD, `offset` elements behind its start."""
    groups, dg = (1, d) if c == 0 else (c, d // c)
    buffer = torch.full((offset + groups * n * (dg + pad),), GUARD, dtype=dtype, device=dev())
    x = buffer[offset:].view(groups, n, dg + pad)[:, :, :dg]
    if values is not None:
        x.copy_(values.to(dtype).view(n, groups, dg).permute(1, 0, 2))
    return buffer, (x[0] if c == 0 else x)


def rows_of(x):
    return x if x.dim() == 2 else x.permute(1, 0, 2).reshape(x.shape[1], -1)


def untouched(buffer, x):
    """Whether everything of the buffer outside the view still holds GUARD."""
    mask = torch.ones_like(buffer, dtype=torch.bool)
    mask.as_strided(x.shape, x.stride(), x.storage_offset()).fill_(False)
    return bool((buffer[mask] == GUARD).all())


def lookup_ref(table, ids, scale, dtype):
    ids = torch.as_tensor(ids, device=dev()).long()
    known = (ids >= 0) & (ids < len(table))
    return torch.where(known[:, None], table.float()[ids.clamp(0, len(table) - 1)] * scale, torch.zeros((), device=dev())).to(dtype)


def grad_ref(dx, ids, vocab, scale):
    """(gradient, sum of absolute values) in float64, on the host."""
    ids = torch.as_tensor(ids).long().cpu()
    known = (ids >= 0) & (ids < vocab)
    x = rows_of(dx).double().cpu()[known]
    out = torch.zeros((vocab, x.shape[1]), dtype=torch.float64)
    return out.index_add(0, ids[known], x) * scale, out.index_add(0, ids[known], x.abs()) * abs(scale)


@pytest.mark.parametrize("n,vocab,d,c,table_type,dtype,ids_type,kind,pad,offset", [
    (1, 1, 1, 0, F32, F32, torch.int32, "one", 0, 0),
    (1, 7, 64, 2, F32, BF16, torch.int64, "mixed", 0, 0),
    (3, 2, 3, 0, BF16, BF16, torch.int32, "mixed", 2, 1),
    (100, 5, 5, 0, F32, F32, torch.int64, "mixed", 0, 3),
    (257, 40, 64, 2, F32, F32, torch.int32, "common", 0, 0),
    (1001, 300, 77, 0, BF16, F32, torch.int32, "mixed", 1, 1),
    (1001, 300, 77, 0, F32, BF16, torch.int64, "mixed", 1, 1),
    (1001, 300, 77, 0, BF16, BF16, torch.int64, "mixed", 3, 1),
    (5000, 97, 256, 4, F32, F32, torch.int32, "common", 0, 0),
    (5000, 97, 256, 8, BF16, BF16, torch.int32, "mixed", 0, 0),
    (4097, 50_021, 192, 3, F32, F32, torch.int64, "distinct", 4, 2),
    (333, 11, 2052, 0, F32, F32, torch.int32, "mixed", 0, 0),
    (17, 11, 9000, 2, BF16, F32, torch.int32, "mixed", 0, 0),
    (9, 4, 131_072, 0, F32, BF16, torch.int32, "mixed", 0, 0),
    (64, 9, 6, 6, F32, F32, torch.int32, "mixed", 0, 0),
    (70, 9, 14, 2, BF16, BF16, torch.int32, "mixed", 0, 0),
    (300, 9, 8, 0, F32, F32, torch.int32, "unknown", 0, 0),
    # odd widths without gaps, in rows and in planes that begin anywhere
    (1, 5, 5, 0, F32, F32, torch.int32, "one", 0, 0),
    (1, 5, 9, 0, BF16, BF16, torch.int32, "one", 0, 0),
    (2, 5, 6, 0, F32, F32, torch.int64, "mixed", 0, 0),
    (1003, 40, 77, 0, F32, F32, torch.int32, "mixed", 0, 0),
    (1003, 40, 77, 0, BF16, F32, torch.int64, "mixed", 0, 0),
    (1003, 40, 301, 0, BF16, BF16, torch.int32, "mixed", 0, 0),
    (1003, 40, 301, 0, F32, BF16, torch.int64, "mixed", 0, 0),
    (20_000, 300, 9, 0, F32, BF16, torch.int32, "common", 0, 0),
    (1000, 40, 231, 3, F32, F32, torch.int32, "mixed", 0, 0),
    (1001, 40, 231, 3, F32, F32, torch.int32, "mixed", 0, 0),
    (1016, 40, 231, 3, BF16, BF16, torch.int32, "mixed", 0, 0),
    (50, 40, 4095, 0, F32, F32, torch.int32, "mixed", 0, 0),
    (50, 40, 4097, 0, F32, F32, torch.int32, "mixed", 0, 0),
    (70, 40, 4095, 0, F32, BF16, torch.int32, "mixed", 0, 0),
])
def test_lookup(n, vocab, d, c, table_type, dtype, ids_type, kind, pad, offset):
    rng = np.random.default_rng(n + d)
    table_buffer, table = plane(vocab, d, 0, table_type, torch.from_numpy(rng.standard_normal((vocab, d))), pad, offset)
    ids = torch.from_numpy(make_ids(kind, n, vocab, rng)).to(ids_type).to(dev())
    buffer, x = plane(n, d, c, dtype, None, pad, offset)
    gsr.gsr_embed_lookup(table, ids, x, 1.7)
    assert torch.equal(rows_of(x), lookup_ref(table, ids, 1.7, dtype))
    assert untouched(buffer, x)


def test_tokens_beyond_32_bits_have_no_embedding():
    ids = torch.tensor([2 ** 32 + 1, 1, -2 ** 32, -2 ** 63, 2 ** 63 - 1, 0], device=dev())
    table = torch.arange(1.0, 9.0, device=dev()).view(2, 4)
    x = torch.full((6, 4), GUARD, device=dev())
    gsr.gsr_embed_lookup(table, ids, x)
    zero = torch.zeros(4, device=dev())
    assert torch.equal(x, torch.stack([zero, table[1], zero, zero, zero, table[0]]))
    dx = torch.arange(24.0, device=dev()).view(6, 4)
    dt = torch.full((2, 4), GUARD, device=dev())
    gsr.gsr_embed_grad(ids, dx, dt)
    assert torch.equal(dt, dx[[5, 1]])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lookup_keeps_infinities_and_nan_to_their_tokens(dtype):
    table = torch.randn(6, 40, device=dev())
    table[2], table[3], table[0] = float("inf"), float("nan"), float("nan")
    ids = torch.tensor([1, 2, 3, -1, 4, 6], dtype=torch.int32, device=dev())
    x = torch.empty((6, 40), dtype=dtype, device=dev())
    gsr.gsr_embed_lookup(table, ids, x, -2.0)
    assert torch.equal(x[[0, 4]], (table[[1, 4]] * -2.0).to(dtype)) and bool((x[1] == float("-inf")).all()) and bool(x[2].isnan().all())
    assert bool((x[[3, 5]] == 0).all())


def test_lookup_rounds_the_product_to_float32_and_then_to_the_plane():
    """(1 + 2^-23) (1 + (2^15 - 1) 2^-23) lies 2^-31 above 1 + 2^-8, to which it rounds in float32: half way between the 16-bit values 1 and
    1 + 2^-7, of which 1 is the even one."""
    table = torch.full((1, 8), 1 + 2.0 ** -23, device=dev())
    ids = torch.zeros(1, dtype=torch.int32, device=dev())
    for dtype, want in ((F32, 1 + 2.0 ** -8), (BF16, 1.0)):
        x = torch.empty((1, 8), dtype=dtype, device=dev())
        gsr.gsr_embed_lookup(table, ids, x, 1 + (2 ** 15 - 1) * 2.0 ** -23)
        assert bool((x.double() == want).all())


# sizes around what one workgroup sorts (4,096) and one stretch of the sort holds (2,048), chunks of 16 to 256 rows, one, two and three passes
# of the sort (vocabularies below 256 and 65,536; 1,024 and 2^20), rows narrower than, as wide as and wider than a piece and a wave
GRADS = [
    (1, 1, 1, 0, F32, torch.int32, "one", 0, 0),
    (1, 3, 64, 2, BF16, torch.int64, "mixed", 0, 0),
    (2, 2, 3, 0, F32, torch.int32, "distinct", 1, 1),
    (16, 5, 7, 0, BF16, torch.int32, "mixed", 2, 1),
    (17, 4, 32, 0, F32, torch.int32, "one", 0, 0),
    (128, 255, 64, 2, F32, torch.int32, "common", 0, 0),
    (129, 256, 77, 0, F32, torch.int64, "mixed", 1, 3),
    (2000, 40, 64, 2, F32, torch.int32, "common", 0, 0),
    (2000, 40, 64, 2, F32, torch.int32, "unknown", 0, 0),
    (2048, 1, 256, 4, F32, torch.int32, "one", 0, 0),
    (2049, 1, 256, 4, F32, torch.int32, "one", 0, 0),
    (2048, 2047, 64, 0, F32, torch.int32, "distinct", 0, 0),
    (2049, 2048, 64, 0, BF16, torch.int32, "common", 0, 0),
    (4095, 65_535, 20, 0, BF16, torch.int64, "distinct", 4, 2),
    (4096, 70_000, 33, 0, BF16, torch.int32, "mixed", 1, 1),
    (4096, 17_000_000, 2, 0, F32, torch.int32, "mixed", 0, 0),
    (4097, 1023, 256, 8, BF16, torch.int32, "common", 0, 0),
    (5000, 1024, 40, 0, F32, torch.int32, "distinct", 0, 0),
    (70_001, 1_048_576, 8, 0, F32, torch.int32, "common", 0, 0),
    (66_000, 511, 24, 0, F32, torch.int32, "mixed", 0, 0),
    (4097, 1, 1, 0, BF16, torch.int32, "one", 0, 0),
    (20_011, 2048, 128, 2, F32, torch.int64, "mixed", 0, 0),
    (65_536, 97, 64, 0, BF16, torch.int32, "common", 0, 0),
    (65_537, 97, 64, 0, F32, torch.int32, "common", 3, 1),
    (70_001, 3, 300, 0, F32, torch.int32, "one", 0, 0),
    (70_001, 300_000, 40, 0, F32, torch.int64, "distinct", 0, 0),
    (70_001, 4_200_000, 4, 0, F32, torch.int32, "mixed", 0, 0),
    (300, 5, 2052, 0, F32, torch.int32, "mixed", 0, 0),
    (90, 5, 9000, 2, BF16, torch.int32, "mixed", 0, 0),
    (40, 3, 131_072, 0, BF16, torch.int32, "mixed", 0, 0),
    (64, 9, 6, 6, F32, torch.int32, "mixed", 0, 0),
    (70, 9, 14, 2, BF16, torch.int32, "mixed", 0, 0),
    (1_100_000, 12, 8, 2, F32, torch.int32, "common", 0, 0),
    (1_100_000, 1, 4, 0, F32, torch.int64, "one", 0, 0),
    (2_200_000, 30, 16, 0, BF16, torch.int64, "common", 0, 0),
    (300_001, 1, 128, 0, F32, torch.int32, "one", 0, 0),
    (150_001, 60, 384, 2, F32, torch.int32, "mixed", 0, 0),
    (600_001, 7, 256, 4, BF16, torch.int32, "common", 0, 0),
    (4096, 6, 8200, 0, BF16, torch.int32, "mixed", 0, 0),
    (4096, 100, 4096, 2, F32, torch.int64, "common", 0, 0),
    (513, 2, 12, 4, F32, torch.int32, "one", 0, 0),
]


@pytest.mark.parametrize("n,vocab,d,c,dtype,ids_type,kind,pad,offset", GRADS)
def test_grad(n, vocab, d, c, dtype, ids_type, kind, pad, offset):
    rng = np.random.default_rng(n + d)
    ids = torch.from_numpy(make_ids(kind, n, vocab, rng)).to(ids_type).to(dev())
    out_buffer, out = plane(vocab, d, 0, F32, None, pad, offset)
    for whole in (True, False):
        values = torch.from_numpy(rng.integers(-8, 9, (n, d)) if whole else rng.standard_normal((n, d))).to(dev())
        buffer, dx = plane(n, d, c, dtype, values, pad, offset)
        gsr.gsr_embed_grad(ids, dx, out, 0.5 if whole else 1.7)
        want, size = grad_ref(dx, ids, vocab, 0.5 if whole else float(np.float32(1.7)))
        got = out.double().cpu()
        if whole:
            assert torch.equal(got, want)
        else:
            assert bool(((got - want).abs() <= 465 * 2.0 ** -24 * size).all()), float(((got - want).abs() / size.clamp(min=1e-300)).max())
            again = torch.full_like(out, GUARD)
            gsr.gsr_embed_grad(ids, dx, again, 1.7)
            assert torch.equal(again, out)
        assert untouched(out_buffer, out)


def test_grad_of_no_rows_is_zero():
    for shape in ((0, 12), (3, 0, 4)):
        out = torch.full((9, 12), GUARD, device=dev())
        gsr.gsr_embed_grad(torch.empty(0, dtype=torch.int32, device=dev()), torch.empty(shape, device=dev()), out)
        assert bool((out == 0).all())
    x = torch.empty((0, 12), device=dev())
    gsr.gsr_embed_lookup(out, torch.empty(0, dtype=torch.int64, device=dev()), x)


def test_grad_keeps_infinities_and_nan_to_their_tokens():
    n, vocab = 5000, 10
    ids = torch.arange(n, device=dev()) % (vocab + 1)          # the last has no embedding
    dx = torch.randn(n, 36, device=dev())
    dx[ids == vocab] = float("nan")
    dx[3], dx[14] = float("inf"), float("nan")                 # tokens 3 and 3
    dx[5] = float("-inf")
    out = torch.empty((vocab, 36), device=dev())
    gsr.gsr_embed_grad(ids, dx, out)
    assert bool(out[3].isnan().all()) and bool((out[5] == float("-inf")).all())
    assert bool(out[[0, 1, 2, 4, 6, 7, 8, 9]].isfinite().all())


def test_grad_is_the_adjoint_and_the_derivative_of_lookup():
    """Whole numbers, so that everything is exact: <dx, lookup(E)> = <grad, E>, and a central difference of the left side along any
    direction is the gradient's product with it (the left side is linear in E)."""
    rng = np.random.default_rng(4)
    n, vocab, d, c, scale = 3001, 50, 96, 3, 2.0
    ids = torch.from_numpy(make_ids("mixed", n, vocab, rng)).to(dev())
    dx = torch.from_numpy(rng.integers(-4, 5, (c, n, d // c)).astype(np.float32)).to(dev())
    table = torch.from_numpy(rng.integers(-16, 17, (vocab, d)).astype(np.float32)).to(dev())
    step = torch.from_numpy(rng.integers(-3, 4, (vocab, d)).astype(np.float32)).to(dev())

    def loss(e):
        x = torch.empty_like(dx)
        gsr.gsr_embed_lookup(e, ids, x, scale)
        return float((x.double() * dx.double()).sum())

    out = torch.empty((vocab, d), device=dev())
    gsr.gsr_embed_grad(ids, dx, out, scale)
    assert loss(table) == float((out.double() * table.double()).sum())
    assert (loss(table + step) - loss(table - step)) / 2 == float((out.double() * step.double()).sum())


def test_offsets_beyond_32_bits():
    """A table, a plane and a gradient of more than 2^31 elements each; whole numbers."""
    n, vocab, d = 8_500_000, 8_400_001, 256
    ids = (torch.arange(n, device=dev()) * 7919) % vocab
    ids[-1], ids[-2], ids[0] = vocab - 1, vocab - 2, vocab - 1
    table = ((torch.arange(vocab, device=dev())[:, None] + torch.arange(d, device=dev())) % 251).to(BF16)
    x = torch.empty((n, d), dtype=BF16, device=dev())
    gsr.gsr_embed_lookup(table, ids, x)
    for a in range(0, n, 1 << 20):
        assert torch.equal(x[a:a + (1 << 20)], table[ids[a:a + (1 << 20)]]), a
    out = torch.empty((vocab, d), dtype=F32, device=dev())
    gsr.gsr_embed_grad(ids, x, out)
    counts = torch.bincount(ids, minlength=vocab)
    for a in range(0, vocab, 1 << 20):
        assert torch.equal(out[a:a + (1 << 20)], table[a:a + (1 << 20)].float() * counts[a:a + (1 << 20), None].float()), a


def test_other_stream_and_captured_calls_that_share_a_workspace():
    """Two captured graphs on one workspace, replayed in turn with new inputs and eager work between, against the eager results."""
    rng = np.random.default_rng(8)
    sizes = [(3000, 60, 64), (70_001, 5000, 32)]
    ws = torch.empty(max(gsr.gsr_embed_grad_workspace(n, v, d) for n, v, d in sizes), dtype=torch.uint8, device=dev())
    side = torch.cuda.Stream()
    calls = []
    for n, vocab, d in sizes:
        t = dict(ids=torch.zeros(n, dtype=torch.int32, device=dev()), table=torch.zeros((vocab, d), device=dev()),
                 x=torch.zeros((n, d), device=dev()), dx=torch.zeros((n, d), device=dev()), out=torch.zeros((vocab, d), device=dev()))

        def call(t=t, ws=ws):
            gsr.gsr_embed_lookup(t["table"], t["ids"], t["x"], 3.0)
            gsr.gsr_embed_grad(t["ids"], t["dx"], t["out"], 3.0, workspace=ws)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        calls.append((t, call, graph, (n, vocab, d)))
    for _ in range(3):
        for t, call, graph, (n, vocab, d) in calls:
            t["ids"].copy_(torch.from_numpy(make_ids("mixed", n, vocab, rng)))
            t["table"].copy_(torch.from_numpy(rng.standard_normal((vocab, d))))
            t["dx"].copy_(torch.from_numpy(rng.standard_normal((n, d))))
            call()
            want = t["x"].clone(), t["out"].clone()
            t["x"].fill_(GUARD)
            t["out"].fill_(GUARD)
            ws.random_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(t["x"], want[0]) and torch.equal(t["out"], want[1])
            assert torch.equal(t["x"], lookup_ref(t["table"], t["ids"], 3.0, F32))


def test_workspace_of_the_largest_graph_serves_smaller_ones():
    """69,631 rows of 256 are cut into chunks of 16 rows, 69,632 into chunks of 32: the smaller call needs more, and finds it."""
    vocab, d, most = 97, 256, 69_632
    ws = torch.empty(gsr.gsr_embed_grad_workspace(most, vocab, d), dtype=torch.uint8, device=dev())
    rng = np.random.default_rng(5)
    for n in (most, most - 1, 16_384, 16_385, 4097, 5):
        ids = torch.from_numpy(make_ids("mixed", n, vocab, rng)).to(dev())
        dx = torch.from_numpy(rng.integers(-8, 9, (n, d)).astype(np.float32)).to(dev())
        out = torch.full((vocab, d), GUARD, device=dev())
        gsr.gsr_embed_grad(ids, dx, out, workspace=ws)
        assert torch.equal(out.double().cpu(), grad_ref(dx, ids, vocab, 1.0)[0]), n


def test_calls_side_by_side_on_two_streams():
    """Two threads' worth of work: calls on two streams with workspaces of their own, many in flight."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    jobs = []
    for i, stream in enumerate(streams):
        n, vocab, d = (9000, 300, 64) if i else (3000, 50, 128)
        rng = np.random.default_rng(i)
        ids = torch.from_numpy(make_ids("common", n, vocab, rng)).to(dev())
        dx = torch.from_numpy(rng.integers(-8, 9, (n, d))).to(dev()).float()
        jobs.append((stream, ids, dx, [torch.full((vocab, d), GUARD, device=dev()) for _ in range(8)], grad_ref(dx, ids, vocab, 1.0)[0]))
    torch.cuda.synchronize()
    for k in range(8):
        for stream, ids, dx, outs, _ in jobs:
            with torch.cuda.stream(stream):
                gsr.gsr_embed_grad(ids, dx, outs[k])
    torch.cuda.synchronize()
    for _, _, _, outs, want in jobs:
        assert all(torch.equal(o.double().cpu(), want) for o in outs)


def test_binding_refuses_what_does_not_fit():
    ids = torch.zeros(4, dtype=torch.int32, device=dev())
    x, table = torch.zeros((4, 8), device=dev()), torch.zeros((3, 8), device=dev())
    for bad in (lambda: gsr.gsr_embed_lookup(table[:, :4], ids, x), lambda: gsr.gsr_embed_lookup(table, ids[:3], x),
                lambda: gsr.gsr_embed_lookup(table, ids.float(), x), lambda: gsr.gsr_embed_lookup(table, ids.cpu(), x),
                lambda: gsr.gsr_embed_lookup(table, ids, x.t()), lambda: gsr.gsr_embed_lookup(table.double(), ids, x),
                lambda: gsr.gsr_embed_lookup(table.cpu(), ids, x), lambda: gsr.gsr_embed_grad(ids, x, table.bfloat16()),
                lambda: gsr.gsr_embed_lookup(table, ids, torch.zeros((3, 4, 8), device=dev())[:, :, :2]),
                lambda: gsr.gsr_embed_lookup(table, ids, torch.zeros((2, 5, 4), device=dev())[:, :4])):
        with pytest.raises((AssertionError, TypeError)):
            bad()
    small = torch.empty(8, dtype=torch.uint8, device=dev())
    gsr.gsr_embed_grad(ids, x, table, workspace=small)       # up to 4,096 rows need none
    with pytest.raises(gsr.GsrError):
        gsr.gsr_embed_grad(ids.repeat(1025), x.repeat(1025, 1), table, workspace=small)
