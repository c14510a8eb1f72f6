"""Performance cases of the operators at the ends of a stack: group norm with an activation over a batch of graphs and its gradient,
activation checkpoints in 8 bits, and softmax cross entropy over many classes without its logits, with its gradient.  Each case has a
plain form in elementary torch operations and the calls of the library; sizes are those of this library's workloads (circuits of 2,000
to 1M nodes, D = 64 to 384) and generic ones.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
BLOCK = 64                      # columns of a row that share the scale of a checkpoint
TINY = 2.0 ** -126


def listed():
    return [
        # Node features of a small design, one graph: launch latency.  Two groups, as the stack's.
        dict(name="norm-2k", op="norm", n=2_000, graphs=1, spare=0, c=2, d=64, layout="planes", groups=2, act="relu", dtype="f32"),
        # The output of the large float32 stack in the planes gsr_step works on.
        dict(name="norm-1m", op="norm", n=1_000_000, graphs=1, spare=0, c=4, d=256, layout="planes", groups=4, act="silu", dtype="f32"),
        # A padded batch of designs of all sizes in 16-bit storage, narrow groups.
        dict(name="norm-batch-bf16", op="norm", n=499_979, graphs=301, spare=979, c=1, d=256, layout="rows", groups=32, act="relu", dtype="bf16"),
        # The gradients of the first and the last; and, on the large stack, both directions as a step of training runs them, what the
        # backward needs of the input kept in 8 bits.
        dict(name="norm-grad-2k", op="norm-grad", n=2_000, graphs=1, spare=0, c=2, d=64, layout="planes", groups=2, act="relu", dtype="f32"),
        dict(name="norm-step8-1m", op="norm-step8", n=1_000_000, graphs=1, spare=0, c=4, d=256, layout="planes", groups=4, act="silu", dtype="f32"),
        dict(name="norm-grad-batch-bf16", op="norm-grad", n=499_979, graphs=301, spare=979, c=1, d=256, layout="rows", groups=32, act="relu", dtype="bf16"),
        # Activations put away in 8 bits and fetched again: a large plane, and rows of odd width in 16-bit storage.
        dict(name="checkpoint-1m", op="checkpoint", n=1_000_000, c=4, d=256, layout="planes", dtype="f32"),
        dict(name="checkpoint-bf16-odd", op="checkpoint", n=249_989, c=1, d=385, layout="rows", dtype="bf16"),
        # Cell types of a small design from its float32 features; then a sample of nodes over a large vocabulary in 16 bits, one in twenty
        # without a class.
        dict(name="class-loss-2k", op="class-loss", n=2_000, classes=40, c=2, d=64, layout="planes", dtype="f32", ids="i32", missing=0.0),
        dict(name="class-loss-32k", op="class-loss", n=32_749, classes=50_021, c=1, d=256, layout="rows", dtype="bf16", ids="i64", missing=0.05),
        # The gradients: float32 features of the paper's width in two groups, and the large vocabulary.
        dict(name="class-grad-f32", op="class-grad", n=8_191, classes=4_099, c=2, d=384, layout="planes", dtype="f32", ids="i32", missing=0.0),
        dict(name="class-grad-32k", op="class-grad", n=32_749, classes=50_021, c=1, d=256, layout="rows", dtype="bf16", ids="i64", missing=0.05),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges above, sizes spread over their logarithm; any width of a row-major plane, whole groups in planes."""
    op = rng.choice(["norm", "norm-grad", "norm-step8", "checkpoint", "class-loss", "class-grad"])
    dtype = rng.choice(["f32", "bf16"])
    if rng.random() < 0.5:
        layout, c = "planes", rng.choice([2, 3, 4, 8])
        d = c * rng.choice([32, 64]) if c == 8 else c * rng.choice([32, 64, 128])
    else:
        layout, c, d = "rows", 1, rng.choice([64, 256, rng.randint(1, 512)])
    case = dict(op=op, c=c, d=d, layout=layout, dtype=dtype)
    if op in ("class-loss", "class-grad"):
        classes = _log_int(rng, 2, 50_000)
        most = 32_749 * 50_021 * 256 if dtype == "bf16" else 32_749 * 50_021 * 32
        n = min(_log_int(rng, 1, 100_000), max(1, most // (classes * d)), 32_749 * 50_021 // classes)
        return dict(case, n=n, classes=classes, ids=rng.choice(["i32", "i64"]), missing=rng.choice([0.0, 0.0, 0.1]))
    n = min(_log_int(rng, 1, 1_000_000), 256_000_000 // d)
    if op == "checkpoint":
        return dict(case, n=n)
    graphs = rng.choice([1, min(n, _log_int(rng, 1, 4_000))])
    spare = rng.randint(0, n // 10) if graphs > 1 else 0
    # a group of two values has a gradient of rounding alone: narrow ones where graphs are long
    groups = rng.choice([g for g in range(1, min(d, 64) + 1) if d % g == 0 and (g == 1 or d // g >= 4 or n >= 64 * graphs)])
    acts = ["none", "silu"] if op == "norm-step8" else ["none", "relu", "silu"]
    return dict(case, n=n, graphs=graphs, spare=spare, groups=groups, act=rng.choice(acts))


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _graph_ptr(case):
    """First rows of the graphs, sizes over three orders of magnitude; some graphs of a batch are empty."""
    rng = random.Random(case["n"] * 1_000_003 + case["graphs"])
    rows = case["n"] - case["spare"]
    shares = [math.exp(rng.uniform(0.0, math.log(1000.0))) for _ in range(case["graphs"])]
    ends, whole, at = [0], sum(shares), 0.0
    for s in shares:
        at += s
        ends.append(min(rows, int(rows * at / whole)))
    ends[-1] = rows
    return torch.tensor(ends, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)  # noqa: E731
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    n, c, d, dtype = case["n"], case["c"], case["d"], DTYPES[case["dtype"]]
    plane = (n, d) if case["layout"] == "rows" else (c, n, d // c)
    s = dict(case=case)
    if case["op"] in ("class-loss", "class-grad"):
        classes = case["classes"]
        # features after a norm, a table in training; the i-th commonest class has a share in proportion to 1 / i
        s["x"] = randn(*plane).to(dtype)
        s["table"] = (randn(classes, d) * (2.0 / math.sqrt(d))).to(dtype)
        s["bias"] = randn(classes)
        rank = torch.exp(rand(n) * math.log(classes + 1.0)).long() - 1
        ids = torch.randperm(classes, generator=gen, device="cuda")[rank.clamp(0, classes - 1)]
        ids[rand(n) < case["missing"]] = -1
        s["targets"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        s["lse"] = torch.empty(n, device="cuda")
        if case["op"] == "class-loss":
            s["loss"] = torch.empty(1, device="cuda")
            return s
        rows = _rows(s["x"])
        for at in range(0, n, 4096):                # what the forward pass left
            s["lse"][at:at + 4096] = torch.logsumexp(rows[at:at + 4096].float() @ s["table"].float().t() + s["bias"], 1)
        s["dx"], s["dtable"], s["dbias"] = torch.empty_like(s["x"]), torch.empty_like(s["table"]), torch.empty_like(s["bias"])
        return s
    # activations of a stack: rows of different size, columns off centre
    s["x"] = (randn(*plane) * torch.exp(0.5 * randn(n, 1)) + 0.3 * randn(plane[-1])).to(dtype)
    if case["op"] == "checkpoint":
        blocks = c * -(-plane[-1] // BLOCK)
        s["codes"] = torch.empty((n, d), dtype=torch.int8, device="cuda")
        s["scales"] = torch.empty((n, blocks), device="cuda")
        s["back"] = torch.empty_like(s["x"])
        return s
    groups, graphs = case["groups"], case["graphs"]
    s["graph_ptr"] = _graph_ptr(case) if graphs > 1 else None
    s["gamma"], s["beta"] = 1.0 + 0.2 * randn(d), 0.2 * randn(d)
    s["y"] = torch.zeros_like(s["x"])
    s["mean"], s["rstd"] = torch.empty((graphs, groups), device="cuda"), torch.empty((graphs, groups), device="cuda")
    if case["op"] == "norm":
        return s
    s["dy"] = randn(*plane).to(dtype)
    s["dx"] = torch.zeros_like(s["x"])
    s["dgamma"], s["dbeta"] = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    if case["op"] == "norm-step8":
        blocks = c * -(-plane[-1] // BLOCK)
        s["codes"] = torch.empty((n, d), dtype=torch.int8, device="cuda")
        s["scales"] = torch.empty((n, blocks), device="cuda")
        return s
    s["mean"], s["rstd"] = _statistics(s, _rows(s["x"]).float())       # what the forward pass left
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------
def _rows(x):
    """[n, d] of a plane in either layout."""
    return x if x.dim() == 2 else x.permute(1, 0, 2).reshape(x.shape[1], -1)


def _plane(rows, like):
    """A plane as `like` of [n, d]."""
    if like.dim() == 2:
        return rows.to(like.dtype)
    return rows.to(like.dtype).reshape(like.shape[1], like.shape[0], like.shape[2]).permute(1, 0, 2).contiguous()


def _graphs(s):
    """(first rows, graph of every row, whether the row has one)."""
    case = s["case"]
    if s["graph_ptr"] is None:
        return torch.tensor([0, case["n"]], device="cuda"), torch.zeros(case["n"], dtype=torch.int64, device="cuda"), None
    ptr = s["graph_ptr"]
    rows = torch.arange(case["n"], device="cuda")
    graph = (torch.searchsorted(ptr, rows, right=True) - 1).clamp(0, case["graphs"] - 1)
    return ptr, graph, (rows >= ptr[0]) & (rows < ptr[-1])


def _group_sums(s, x, ptr):
    """Sums of [n, d] over the rows of every graph and the columns of every group, in 64 bits: up to 256M values in one."""
    per_row = x.reshape(len(x), s["case"]["groups"], -1).sum(2, dtype=torch.float64)
    running = torch.nn.functional.pad(torch.cumsum(per_row.t().contiguous(), 1), (1, 0))
    return (running[:, ptr[1:]] - running[:, ptr[:-1]]).t().contiguous()


def _statistics(s, x):
    case = s["case"]
    ptr, graph, _ = _graphs(s)
    width = case["d"] // case["groups"]
    count = ((ptr[1:] - ptr[:-1]) * width).clamp(min=1)[:, None].double()
    mean = _group_sums(s, x, ptr) / count
    off = x - mean.float()[graph].repeat_interleave(width, 1)
    variance = _group_sums(s, off.square(), ptr) / count
    return mean.float(), (1.0 / (variance + EPS).sqrt()).float()


def _normal(s, x, mean, rstd):
    _, graph, _ = _graphs(s)
    width = s["case"]["d"] // s["case"]["groups"]
    return (x - mean[graph].repeat_interleave(width, 1)) * rstd[graph].repeat_interleave(width, 1)


def _norm(s):
    """y, mean, rstd; rows of no graph keep what y holds."""
    x = _rows(s["x"]).float()
    mean, rstd = _statistics(s, x)
    z = _normal(s, x, mean, rstd) * s["gamma"] + s["beta"]
    act = s["case"]["act"]
    y = z.clamp(min=0.0) if act == "relu" else z * (1.0 / (1.0 + torch.exp(-z))) if act == "silu" else z
    known = _graphs(s)[2]
    if known is not None:
        y = torch.where(known[:, None], y, _rows(s["y"]).float())
    return _plane(y, s["y"]), mean, rstd


def _norm_grad(s, x, mean, rstd):
    ptr, graph, known = _graphs(s)
    case = s["case"]
    width = case["d"] // case["groups"]
    dz = _rows(s["dy"]).float()
    if known is not None:
        dz = dz * known[:, None]
        x = x * known[:, None]
    normal = _normal(s, x, mean, rstd)
    if case["act"] == "relu":                       # which side of zero: in 64 bits
        z = _normal(s, x.double(), mean.double(), rstd.double()) * s["gamma"].double() + s["beta"].double()
        dz = dz * (z > 0.0)
    elif case["act"] == "silu":
        z = normal * s["gamma"] + s["beta"]
        share = 1.0 / (1.0 + torch.exp(-z))
        dz = dz * (share * (1.0 + z * (1.0 - share)))
    dbeta, dgamma = dz.sum(0, dtype=torch.float64).float(), (dz * normal).sum(0, dtype=torch.float64).float()
    h = dz * s["gamma"]
    count = ((ptr[1:] - ptr[:-1]) * width).clamp(min=1)[:, None].double()
    m1 = (_group_sums(s, h, ptr) / count).float()[graph].repeat_interleave(width, 1)
    m2 = (_group_sums(s, h * normal, ptr) / count).float()[graph].repeat_interleave(width, 1)
    dx = rstd[graph].repeat_interleave(width, 1) * (h - m1 - normal * m2)
    if known is not None:
        dx = torch.where(known[:, None], dx, _rows(s["dx"]).float())
    return {"dx": _plane(dx, s["dx"]), "dgamma": dgamma, "dbeta": dbeta}


def _blocks(x):
    """The columns of every group in blocks, the last one filled up with zeros: [.., blocks, BLOCK]."""
    short = -x.shape[-1] % BLOCK
    return torch.nn.functional.pad(x, (0, short)).unflatten(-1, (-1, BLOCK))


def _through_8_bits(x):
    """What a plane's checkpoint stands for, in float32; the side of a border between two codes on which a value lies in 64 bits."""
    blocks = _blocks(x.float())
    top = blocks.abs().amax(-1, keepdim=True).clamp(min=127.0 * TINY)
    codes = torch.round(blocks.double() * 127.0 / top.double()).float()
    return (codes * (top / 127.0)).flatten(-2)[..., :x.shape[-1]]


def _class_gradient(s):
    """dz of the mean loss for the rows with a class, zero for the others."""
    targets = s["targets"].long()
    known = (targets >= 0) & (targets < s["case"]["classes"])
    z = _rows(s["x"]).float() @ s["table"].float().t()
    z += s["bias"]
    z -= s["lse"][:, None]
    p = torch.exp_(z)
    p[torch.arange(len(p), device="cuda"), targets.clamp(0, s["case"]["classes"] - 1)] -= known.float()
    p *= (known / known.sum().clamp(min=1))[:, None].float()
    return p


def _plain(s):
    op = s["case"]["op"]
    if op == "norm":
        y, mean, rstd = _norm(s)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm-grad":
        return _norm_grad(s, _rows(s["x"]).float(), s["mean"], s["rstd"])
    if op == "norm-step8":
        y, mean, rstd = _norm(s)
        return {"y": y, "mean": mean, "rstd": rstd, **_norm_grad(s, _rows(_through_8_bits(s["x"])), mean, rstd)}
    if op == "checkpoint":
        return _through_8_bits(s["x"]).to(s["x"].dtype)
    if op == "class-loss":
        targets = s["targets"].long()
        known = (targets >= 0) & (targets < s["case"]["classes"])
        z = _rows(s["x"]).float() @ s["table"].float().t()
        z += s["bias"]
        at = z.gather(1, targets.clamp(0, s["case"]["classes"] - 1)[:, None])[:, 0]
        top = z.amax(1)
        z -= top[:, None]
        lse = top + torch.log(torch.exp_(z).sum(1))
        loss = torch.where(known, lse - at, 0.0).sum(dtype=torch.float64) / known.sum().clamp(min=1)
        return {"loss": loss.float().reshape(1), "lse": lse}
    dz = _class_gradient(s)
    return {"dx": _plane(dz @ s["table"].float(), s["dx"]), "dtable": (dz.t() @ _rows(s["x"]).float()).to(s["dtable"].dtype),
            "dbias": dz.sum(0, dtype=torch.float64).float()}


def run(s):
    if not own:
        return _plain(s)
    import paper_2603_27156_amd as gsr
    case = s["case"]
    op = case["op"]
    if op == "checkpoint":
        gsr.gsr_checkpoint_save(s["x"], s["codes"], s["scales"])
        gsr.gsr_checkpoint_load(s["codes"], s["scales"], s["back"])
        return s["back"]
    if op == "class-loss":
        gsr.gsr_class_loss(s["x"], s["table"], s["targets"], s["loss"], s["lse"], bias=s["bias"])
        return {"loss": s["loss"], "lse": s["lse"]}
    if op == "class-grad":
        gsr.gsr_class_grad(s["x"], s["table"], s["targets"], s["lse"], dx_out=s["dx"], dtable_out=s["dtable"], bias=s["bias"], dbias_out=s["dbias"])
        return {"dx": s["dx"], "dtable": s["dtable"], "dbias": s["dbias"]}
    act = {"none": gsr.GSR_ACT_NONE, "relu": gsr.GSR_ACT_RELU, "silu": gsr.GSR_ACT_SILU}[case["act"]]
    affine = dict(gamma=s["gamma"], beta=s["beta"], act=act, graph_ptr=s["graph_ptr"])
    if op == "norm":
        gsr.gsr_group_norm(s["x"], s["y"], s["mean"], s["rstd"], eps=EPS, **affine)
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    grads = dict(dgamma_out=s["dgamma"], dbeta_out=s["dbeta"], **affine)
    out = {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if op == "norm-grad":
        gsr.gsr_group_norm_grad(s["dy"], s["mean"], s["rstd"], s["dx"], x=s["x"], **grads)
        return out
    gsr.gsr_group_norm(s["x"], s["y"], s["mean"], s["rstd"], eps=EPS, codes_out=s["codes"], scales_out=s["scales"], **affine)
    gsr.gsr_group_norm_grad(s["dy"], s["mean"], s["rstd"], s["dx"], codes=s["codes"], scales=s["scales"], **grads)
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"], **out}


def work(case):
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    op, n, c, d, b = case["op"], case["n"], case["c"], case["d"], size[case["dtype"]]
    if op in ("class-loss", "class-grad"):
        classes = case["classes"]
        inputs = (n + classes) * d * b + n * size[case["ids"]] + classes * 4
        if op == "class-loss":
            return {"bytes": inputs + n * 4 + 4, "flops": 2 * n * classes * d}
        return {"bytes": inputs + n * 4 + (n + classes) * d * b + classes * 4, "flops": 6 * n * classes * d}
    scales = n * c * -(-(d // c) // BLOCK) * 4
    if op == "checkpoint":
        return {"bytes": 2 * (n * d * (b + 1) + scales), "flops": 4 * n * d}
    rows, stats = n - case["spare"], case["graphs"] * case["groups"] * 8
    forward, backward = rows * d * 2 * b + stats + d * 8, rows * d * 3 * b + stats + d * 16
    if op == "norm":
        return {"bytes": forward, "flops": 10 * rows * d}
    if op == "norm-grad":
        return {"bytes": backward, "flops": 20 * rows * d}
    return {"bytes": forward + backward - rows * d * b + 2 * (rows * d + scales), "flops": 34 * rows * d}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _rows64(x):
    return x.double() if x.dim() == 2 else torch.cat(list(x), 1).double()


def _like(rows, plane):
    return rows if plane.dim() == 2 else torch.stack(rows.chunk(plane.shape[0], 1))


def _spans(s):
    ptr = [0, s["case"]["n"]] if s["graph_ptr"] is None else s["graph_ptr"].tolist()
    return [(i, a, b) for i, (a, b) in enumerate(zip(ptr, ptr[1:])) if b > a]


def _exact_statistics(s, x):
    """Mean and 1 / sqrt(variance + eps) of every graph and group; an empty graph has the mean 0 and the variance 0."""
    groups = s["case"]["groups"]
    mean = torch.zeros((s["case"]["graphs"], groups), dtype=torch.float64, device="cuda")
    rstd = torch.full_like(mean, 1.0 / math.sqrt(EPS))
    for i, a, b in _spans(s):
        part = x[a:b].unflatten(1, (groups, -1))
        variance, m = torch.var_mean(part, dim=(0, 2), correction=0)
        mean[i], rstd[i] = m, torch.rsqrt(variance + EPS)
    return mean, rstd


def _exact_norm(s, x, mean, rstd):
    y = _rows64(s["y"])
    gamma, beta = s["gamma"].double(), s["beta"].double()
    for i, a, b in _spans(s):
        part = (x[a:b].unflatten(1, (s["case"]["groups"], -1)) - mean[i][:, None]) * rstd[i][:, None]
        z = torch.addcmul(beta, part.flatten(1), gamma)
        y[a:b] = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * torch.sigmoid(t)}[s["case"]["act"]](z)
    return y


def _exact_norm_grad(s, x, mean, rstd):
    case = s["case"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    dy, dx = _rows64(s["dy"]), _rows64(s["dx"])
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
    for i, a, b in _spans(s):
        normal = ((x[a:b].unflatten(1, (case["groups"], -1)) - mean[i][:, None]) * rstd[i][:, None]).flatten(1)
        z = normal * gamma + beta
        if case["act"] == "relu":
            slope = torch.heaviside(z, torch.zeros((), dtype=torch.float64, device="cuda"))
        elif case["act"] == "silu":
            slope = torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        else:
            slope = torch.ones_like(z)
        dz = dy[a:b] * slope
        dgamma += torch.einsum("nd,nd->d", dz, normal)
        dbeta += dz.sum(0)
        h, v = (dz * gamma).unflatten(1, (case["groups"], -1)), normal.unflatten(1, (case["groups"], -1))
        h = h - h.mean((0, 2), keepdim=True) - v * (h * v).mean((0, 2), keepdim=True)
        dx[a:b] = (h * rstd[i][:, None]).flatten(1)
    return {"dx": _like(dx, s["dx"]), "dgamma": dgamma, "dbeta": dbeta}


def _exact_8_bits(x):
    """Every row's blocks of a group, one block of columns after the other."""
    x = x.double()
    out = torch.empty_like(x)
    for a in range(0, x.shape[-1], BLOCK):
        part = x[..., a:a + BLOCK]
        top = torch.linalg.vector_norm(part, ord=math.inf, dim=-1, keepdim=True).clamp(min=127.0 * TINY)
        out[..., a:a + BLOCK] = torch.round(127.0 * part / top) * top / 127.0
    return out


def _exact_class(case, s):
    x, table, bias, targets = _rows64(s["x"]), s["table"].double(), s["bias"].double(), s["targets"].long()
    known = (targets >= 0) & (targets < case["classes"])
    count = max(1, int(known.sum()))
    lse, loss = torch.empty(case["n"], dtype=torch.float64, device="cuda"), 0.0
    dx, dtable, dbias = torch.zeros_like(x), torch.zeros_like(table), torch.zeros_like(bias)
    for a in range(0, case["n"], 4096):
        z = torch.addmm(bias, x[a:a + 4096], table.t())
        k, t = known[a:a + 4096], targets[a:a + 4096]
        if case["op"] == "class-loss":
            lse[a:a + 4096] = torch.logsumexp(z, 1)
            loss += float((lse[a:a + 4096] - z.gather(1, t.clamp(0, case["classes"] - 1)[:, None])[:, 0])[k].sum())
            continue
        dz = torch.exp(z - s["lse"][a:a + 4096, None].double())
        dz.scatter_add_(1, t.clamp(0, case["classes"] - 1)[:, None], torch.full((len(z), 1), -1.0, dtype=torch.float64, device="cuda"))
        dz = dz * (k[:, None] / count)
        dx[a:a + 4096] = dz @ table
        dtable += dz.t() @ x[a:a + 4096]
        dbias += dz.sum(0)
    if case["op"] == "class-loss":
        return {"loss": torch.tensor([loss / count], dtype=torch.float64), "lse": lse}
    return {"dx": _like(dx, s["dx"]), "dtable": dtable, "dbias": dbias}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "checkpoint":
        return _exact_8_bits(s["x"])
    if op in ("class-loss", "class-grad"):
        return _exact_class(case, s)
    x = _rows64(s["x"])
    if op == "norm-grad":
        return _exact_norm_grad(s, x, s["mean"].double(), s["rstd"].double())
    mean, rstd = _exact_statistics(s, x)
    out = {"y": _like(_exact_norm(s, x, mean, rstd), s["y"]), "mean": mean, "rstd": rstd}
    if op == "norm-step8":
        out.update(_exact_norm_grad(s, _rows64(_exact_8_bits(s["x"])), mean, rstd))
    return out
