"""Performance cases of the operators around a training step: node embeddings and their gradient, the norm of a list of
gradients, clipping, and Adam over a list of tensors.  Each case has a plain form in elementary torch operations and the call of
the library; sizes are those of this library's workloads (circuits of 2,000 to 1M nodes, D = 64 to 256, stacks of up to 112 layers)
and, for the lists, generic ones up to 400M elements.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ADAM = dict(t=7, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=1e-2)
CLIP_EPS = 1e-6


def listed():
    return [
        # Node features of a small design looked up by cell type: launch latency is all there is.
        dict(name="lookup-2k", op="lookup", n=2_000, vocab=40, c=2, d=64, layout="planes", table="f32", dtype="f32", ids="i32", missing=0.0),
        # The features of the large float32 stack, in the planes gsr_step works on.
        dict(name="lookup-1m", op="lookup", n=1_000_000, vocab=4_099, c=4, d=256, layout="planes", table="f32", dtype="f32", ids="i32", missing=0.0),
        # 16-bit storage at an odd size, a large vocabulary, 64-bit tokens, one in twenty of them without an embedding.
        dict(name="lookup-bf16-odd", op="lookup", n=499_979, vocab=50_021, c=1, d=256, layout="rows", table="bf16", dtype="bf16", ids="i64", missing=0.05),
        # The gradients of the same three: few nodes; a million nodes of a hundred cell types (one row in six is of the commonest);
        # 16-bit gradients to a large, mostly rare vocabulary.
        dict(name="embed-grad-2k", op="embed-grad", n=2_000, vocab=40, c=2, d=64, layout="planes", dtype="f32", ids="i32", missing=0.0),
        dict(name="embed-grad-1m", op="embed-grad", n=1_000_000, vocab=97, c=4, d=256, layout="planes", dtype="f32", ids="i32", missing=0.0),
        dict(name="embed-grad-bf16-odd", op="embed-grad", n=499_979, vocab=50_021, c=1, d=256, layout="rows", dtype="bf16", ids="i64", missing=0.05),
        # The gradients of a small design's stack, for the log: latency.  And those of a large generic model, 16 bits wide.
        dict(name="norm-step-2k", op="norm", tensors=7, total=8_192 + 64 + 1 + 2_560, dtype="f32", packed=False),
        dict(name="norm-400m", op="norm", tensors=300, total=400_000_000, dtype="bf16", packed=False),
        # A stack of 112 layers with a matrix tensor each, head and embedding: many small tensors.  And a large model's gradients out of
        # one buffer, odd sizes behind each other.
        dict(name="clip-112-layers", op="clip", tensors=115, total=2_884_609, dtype="f32", out="f32", packed=False, clipped=True),
        dict(name="clip-200m", op="clip", tensors=333, total=201_326_611, dtype="f32", out="f32", packed=True, clipped=True),
        # The clipped update of the same stack, norm included, and of a large model with 16-bit gradients.
        dict(name="adam-112-layers", op="adam", tensors=115, total=2_884_609, dtype="f32", packed=False, clipped=True),
        dict(name="adam-120m", op="adam", tensors=260, total=120_000_000, dtype="bf16", packed=False, clipped=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges above, sizes spread over their logarithm; any width of a row-major plane, whole groups in planes."""
    op = rng.choice(["lookup", "embed-grad", "embed-grad", "norm", "clip", "adam"])
    dtype = rng.choice(["f32", "f32", "bf16"])
    if op in ("lookup", "embed-grad"):
        if rng.random() < 0.5:
            layout, c = "planes", rng.choice([2, 3, 4, 8])
            d = c * rng.choice([32, 64]) if c == 8 else c * rng.choice([32, 64, 128])
        else:
            layout, c, d = "rows", 1, rng.choice([64, 256, rng.randint(1, 512)])
        n = min(_log_int(rng, 1, 1_000_000), 256_000_000 // d)
        case = dict(op=op, n=n, vocab=_log_int(rng, 2, 200_000), c=c, d=d, layout=layout, dtype=dtype, ids=rng.choice(["i32", "i64"]),
                    missing=rng.choice([0.0, 0.0, 0.1]))
        return dict(case, table=rng.choice(["f32", "bf16"])) if op == "lookup" else case
    total = _log_int(rng, 1_000, 100_000_000)
    case = dict(op=op, tensors=min(_log_int(rng, 1, 400), total), total=total, dtype=dtype, packed=rng.random() < 0.4)
    if op == "norm":
        return case
    case["clipped"] = rng.random() < 0.8
    return dict(case, out=rng.choice([dtype, "f32"])) if op == "clip" else case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _sizes(case):
    """Elements of every tensor: spread over three orders of magnitude, as matrices, biases and scalars of a model are."""
    rng = random.Random(case["tensors"] * 1_000_003 + case["total"])
    shares = [math.exp(rng.uniform(0.0, math.log(1000.0))) for _ in range(case["tensors"])]
    spare, whole = case["total"] - case["tensors"], sum(shares)
    sizes = [1 + int(spare * s / whole) for s in shares]
    sizes[0] += case["total"] - sum(sizes)
    return sizes


def _views(case, values, dtype):
    """(buffer, tensors): the tensors one behind the other, or each from a multiple of 64 elements on with zeros between."""
    sizes, step = _sizes(case), 1 if case["packed"] else 64
    places = np.cumsum([0] + [-(-k // step) * step for k in sizes])
    flat = torch.zeros(int(places[-1]), dtype=dtype, device="cuda")
    tensors = [flat[int(p):int(p) + k] for p, k in zip(places, sizes)]
    torch._foreach_copy_(tensors, list(values.split(sizes)))
    return flat, tensors


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)  # noqa: E731
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    s = dict(case=case)
    if case["op"] in ("lookup", "embed-grad"):
        n, vocab, c, d = case["n"], case["vocab"], case["c"], case["d"]
        # the i-th commonest token has a share in proportion to 1 / i; which tokens are common is drawn too
        rank = torch.exp(rand(n) * math.log(vocab + 1.0)).long() - 1
        ids = torch.randperm(vocab, generator=gen, device="cuda")[rank.clamp(0, vocab - 1)]
        ids[rand(n) < case["missing"]] = -1
        s["ids"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        s["scale"] = math.sqrt(d)
        plane = (n, d) if case["layout"] == "rows" else (c, n, d // c)
        if case["op"] == "lookup":
            s["table"] = (randn(vocab, d) * 0.02).to(DTYPES[case["table"]])
            s["x"] = torch.empty(plane, dtype=DTYPES[case["dtype"]], device="cuda")
        else:
            s["dx"] = (randn(*plane) / n).to(DTYPES[case["dtype"]])
            s["dtable"] = torch.empty((vocab, d), dtype=torch.float32, device="cuda")
        return s
    total = case["total"]
    values = randn(total) * torch.exp(3.0 * rand(1).float())        # gradients of one step, their scale drawn with them
    s["flat_g"], s["g"] = _views(case, values, DTYPES[case["dtype"]])
    s["norm"] = torch.zeros(1, dtype=torch.float32, device="cuda")
    if case["op"] == "norm":
        return s
    s["max_norm"] = 1.0 if case["clipped"] else 100.0 * math.sqrt(total)
    if case["op"] == "clip":
        s["flat_out"], s["out"] = _views(case, torch.zeros(total, device="cuda"), DTYPES[case["out"]])
        return s
    # weights and Adam's state in the middle of a training run with clipped gradients
    typical = 1.0 / math.sqrt(total) if case["clipped"] else 1.0
    s["flat_w"], s["w"] = _views(case, randn(total) * 0.02, torch.float32)
    s["flat_m"], s["m"] = _views(case, randn(total) * (0.3 * typical), torch.float32)
    s["flat_v"], s["v"] = _views(case, randn(total).square() * typical ** 2, torch.float32)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------
def _rows(x):
    """[n, d] of a plane in either layout."""
    return x if x.dim() == 2 else x.permute(1, 0, 2).reshape(x.shape[1], -1)


def _norm(flat):
    return flat.square().sum(dtype=torch.float64).sqrt().float().reshape(1)


def _coefficient(norm, max_norm):
    return (max_norm / (norm + CLIP_EPS)).clamp(max=1.0)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "lookup":
        ids, table, x = s["ids"].long(), s["table"], s["x"]
        known = (ids >= 0) & (ids < len(table))
        rows = (table[ids.clamp(0, len(table) - 1)].float() * s["scale"]).masked_fill(~known[:, None], 0.0)
        return rows.to(x.dtype) if x.dim() == 2 else rows.to(x.dtype).reshape(len(ids), case["c"], -1).permute(1, 0, 2).contiguous()
    if op == "embed-grad":
        # running sums over the rows in the order of their tokens, taken where a token ends less where it begins
        ids, vocab = s["ids"].long(), case["vocab"]
        ids, order = torch.sort(torch.where((ids >= 0) & (ids < vocab), ids, vocab))
        columns = _rows(s["dx"])[order].t().double()                         # up to a million rows in one sum
        sums = torch.nn.functional.pad(torch.cumsum(columns.contiguous(), 1), (1, 0))
        ends = torch.searchsorted(ids, torch.arange(-1, vocab, device="cuda"), right=True)
        return ((sums[:, ends[1:]] - sums[:, ends[:-1]]) * s["scale"]).float().t().contiguous()
    g = torch.cat(s["g"]).float()
    norm = _norm(g)
    if op == "norm":
        return norm
    g = g * _coefficient(norm, s["max_norm"])
    sizes = [len(t) for t in s["g"]]
    if op == "clip":
        torch._foreach_copy_(s["out"], list(g.to(s["flat_out"].dtype).split(sizes)))
        return {"norm": norm, "out": s["flat_out"]}
    a = ADAM
    w, m, v = torch.cat(s["w"]), torch.cat(s["m"]), torch.cat(s["v"])
    g = g + a["weight_decay"] * w
    m = a["beta1"] * m + (1.0 - a["beta1"]) * g
    v = a["beta2"] * v + (1.0 - a["beta2"]) * g.square()
    w = w - a["lr"] * (m / (1.0 - a["beta1"] ** a["t"])) / ((v / (1.0 - a["beta2"] ** a["t"])).sqrt() + a["eps"])
    torch._foreach_copy_(s["w"] + s["m"] + s["v"], list(w.split(sizes)) + list(m.split(sizes)) + list(v.split(sizes)))
    return {"norm": norm, "w": s["flat_w"], "m": s["flat_m"], "v": s["flat_v"]}


def run(s):
    if not own:
        return _plain(s)
    import paper_2603_27156_amd as gsr
    op = s["case"]["op"]
    if op == "lookup":
        gsr.gsr_embed_lookup(s["table"], s["ids"], s["x"], s["scale"])
        return s["x"]
    if op == "embed-grad":
        gsr.gsr_embed_grad(s["ids"], s["dx"], s["dtable"], s["scale"])
        return s["dtable"]
    if op == "norm":
        gsr.gsr_grad_norm(s["g"], s["norm"])
        return s["norm"]
    if op == "clip":
        gsr.gsr_grad_clip(s["g"], s["max_norm"], s["norm"], out=s["out"])
        return {"norm": s["norm"], "out": s["flat_out"]}
    gsr.gsr_grad_norm(s["g"], s["norm"])
    gsr.gsr_adam_update_list(s["w"], s["g"], s["m"], s["v"], norm=s["norm"], max_norm=s["max_norm"], **ADAM)
    return {"norm": s["norm"], "w": s["flat_w"], "m": s["flat_m"], "v": s["flat_v"]}


def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    op = case["op"]
    if op in ("lookup", "embed-grad"):
        n, vocab, d = case["n"], case["vocab"], case["d"]
        known = n * (1.0 - case["missing"])
        if op == "embed-grad":
            return {"bytes": n * size[case["ids"]] + known * d * size[case["dtype"]] + vocab * d * 4, "flops": known * d}
        share = np.diff(np.log(np.arange(1, vocab + 2))) / math.log(vocab + 1)
        distinct = float((1.0 - np.exp(known * np.log1p(-share))).sum())
        return {"bytes": n * size[case["ids"]] + distinct * d * size[case["table"]] + n * d * size[case["dtype"]], "flops": n * d}
    total, b = case["total"], size[case["dtype"]]
    if op == "norm":
        return {"bytes": total * b, "flops": 2 * total}
    if op == "clip":
        return {"bytes": total * (b + size[case["out"]]), "flops": 3 * total}
    return {"bytes": total * (b + 24), "flops": 18 * total}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _exact_lookup(s):
    table = torch.cat([torch.zeros((1, s["table"].shape[1]), dtype=torch.float64, device="cuda"), s["table"].double()])
    rows = table.index_select(0, s["ids"].long() + 1) * s["scale"]       # -1, no token, is the row of zeros in front
    return rows if s["x"].dim() == 2 else torch.stack(rows.chunk(s["case"]["c"], dim=1))


def _exact_embed_grad(s):
    """Every row added to its token's, one after the other."""
    ids = s["ids"].long()
    rows = s["dx"] if s["dx"].dim() == 2 else torch.cat(list(s["dx"]), 1)
    sums = torch.zeros(s["dtable"].shape, dtype=torch.float64, device="cuda")
    return sums.index_add_(0, ids[ids >= 0], rows[ids >= 0].double()).mul_(s["scale"])


def _exact_list(case, s):
    buffer = s["flat_g"].double()                                    # zeros lie between the tensors
    norm = torch.linalg.vector_norm(buffer).reshape(1)
    if case["op"] == "norm":
        return norm
    c = min(1.0, s["max_norm"] / (float(norm) + CLIP_EPS))
    if case["op"] == "clip":
        return {"norm": norm, "out": buffer * c}
    a = ADAM
    m, v, w = s["flat_m"].double(), s["flat_v"].double(), s["flat_w"].double()
    g = torch.add(buffer * c, w, alpha=a["weight_decay"])
    m = torch.lerp(m, g, 1.0 - a["beta1"])
    v = torch.lerp(v, g * g, 1.0 - a["beta2"])
    root = torch.sqrt(v / (1.0 - a["beta2"] ** a["t"])) + a["eps"]
    return {"norm": norm, "w": w - (a["lr"] / (1.0 - a["beta1"] ** a["t"])) * m / root, "m": m, "v": v}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "lookup":
        return _exact_lookup(s)
    return _exact_embed_grad(s) if case["op"] == "embed-grad" else _exact_list(case, s)
