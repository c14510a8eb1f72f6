"""The ends of a stack together: embeddings, a group norm whose input is kept in 8 bits, reversible layers, a group norm, cross entropy over the types of the
nodes with the table of the embeddings, and all the way back; on the library's own graph and layer calls, against the same chain taken apart."""
import numpy as np
import pytest
import torch

import paper_2603_27156_amd as gsr
from paper_2603_27156_amd import synth

pytestmark = pytest.mark.gpu


def dev():
    return torch.device("cuda:0")


class Model:
    def __init__(self, dtype, seed=0, k=None):
        w = synth.scaled(synth.workload(0), 900)
        inp = synth.make_inputs(w, seed)
        self.n, self.d, self.c, self.types, self.groups = w.n, w.d, w.c, 40, 4
        self.graph = gsr.gsr_graph_create(inp.rowptr, inp.colidx)
        self.cfg = gsr.Config(n=w.n, d=w.d, c=w.c, k=k or w.k, layout=gsr.GSR_LAYOUT_GROUP_PLANAR, dtype=gsr.GSR_F32 if dtype == torch.float32 else gsr.GSR_BF16)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen, device=dev())  # noqa: E731
        self.dtype = dtype
        self.table = rand(self.types, self.d).to(dtype)
        self.w = [torch.from_numpy(inp.weights[l]).to(dev()).contiguous() for l in range(2)]
        self.gamma = [1.0 + 0.1 * rand(self.d) for _ in range(2)]
        self.beta = [0.1 * rand(self.d) for _ in range(2)]
        self.bias = 0.1 * rand(self.types)
        self.ids = torch.randint(0, self.types, (self.n,), generator=gen, device=dev(), dtype=torch.int32)
        self.targets = torch.randint(0, self.types, (self.n,), generator=gen, device=dev(), dtype=torch.int32)
        self.targets[torch.rand(self.n, generator=gen, device=dev()) > 0.3] = -1        # the others are not asked for
        self.ptr = torch.tensor([0, 300, self.n], device=dev())
        self.ws = torch.empty(gsr.gsr_workspace_size(self.graph, self.cfg)[0], dtype=torch.uint8, device=dev())

    def plane(self):
        return torch.empty((self.c, self.n, self.d // self.c), dtype=self.dtype, device=dev())

    def norm(self, i, x, y, mean, rstd, **kw):
        gsr.gsr_group_norm(x, y, mean, rstd, gamma=self.gamma[i], beta=self.beta[i], act=gsr.GSR_ACT_SILU, graph_ptr=self.ptr, **kw)

    def buffers(self):
        z = lambda *s: torch.zeros(s, device=dev())  # noqa: E731
        o = dict(loss=z(1), lse=z(self.n), dtable=torch.zeros_like(self.table), dbias=z(self.types), dembed=z(self.types, self.d), h=self.plane(), g=self.plane(),
                 dx=self.plane(), x0=self.plane(), codes=torch.zeros((self.n, self.d), dtype=torch.int8, device=dev()),
                 scales=z(self.n, gsr.gsr_checkpoint_blocks(self.d, self.c)))
        for i in range(2):
            o.update({f"mean{i}": z(2, self.groups), f"rstd{i}": z(2, self.groups), f"dgamma{i}": z(self.d), f"dbeta{i}": z(self.d), f"dw{i}": torch.zeros_like(self.w[i])})
        return o

    def step(self, o):
        """One training step; the stack keeps nothing, the first norm its input in 8 bits."""
        gsr.gsr_embed_lookup(self.table, self.ids, o["h"])
        self.norm(0, o["h"], o["h"], o["mean0"], o["rstd0"], codes_out=o["codes"], scales_out=o["scales"])       # in place
        o["x0"].copy_(o["h"])
        for l in range(2):
            gsr.gsr_layer_forward(self.graph, self.cfg, self.w[l], o["h"], workspace=self.ws)
        self.norm(1, o["h"], o["g"], o["mean1"], o["rstd1"])
        gsr.gsr_class_loss(o["g"], self.table, self.targets, o["loss"], o["lse"], bias=self.bias)
        gsr.gsr_class_grad(o["g"], self.table, self.targets, o["lse"], dx_out=o["dx"], dtable_out=o["dtable"], bias=self.bias, dbias_out=o["dbias"])
        gsr.gsr_group_norm_grad(o["dx"], o["mean1"], o["rstd1"], o["dx"], x=o["h"], gamma=self.gamma[1], beta=self.beta[1], act=gsr.GSR_ACT_SILU,
                                graph_ptr=self.ptr, dgamma_out=o["dgamma1"], dbeta_out=o["dbeta1"])
        for l in (1, 0):
            gsr.gsr_layer_backward(self.graph, self.cfg, self.w[l], o["h"], o["dx"], o[f"dw{l}"], workspace=self.ws)
        gsr.gsr_group_norm_grad(o["dx"], o["mean0"], o["rstd0"], o["dx"], codes=o["codes"], scales=o["scales"], gamma=self.gamma[0], beta=self.beta[0],
                                act=gsr.GSR_ACT_SILU, graph_ptr=self.ptr, dgamma_out=o["dgamma0"], dbeta_out=o["dbeta0"])
        gsr.gsr_embed_grad(self.ids, o["dx"], o["dembed"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_against_the_same_step_taken_apart(dtype):
    m = Model(dtype)
    o = m.buffers()
    m.step(o)
    rows = lambda p: p.permute(1, 0, 2).reshape(m.n, m.d).double()                                  # noqa: E731
    groups = lambda v: v.reshape(-1, m.groups, m.d // m.groups)                                     # noqa: E731
    of_rows = lambda v: torch.cat([v[:1].expand(300, -1), v[1:].expand(m.n - 300, -1)]).double().repeat_interleave(m.d // m.groups, 1)     # noqa: E731
    u = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    # embeddings and the first norm: off by roundings of values of size 4 to 8
    x = m.table.double()[m.ids.long()]
    xh = (x - of_rows(o["mean0"])) * of_rows(o["rstd0"])
    z = xh * m.gamma[0].double() + m.beta[0].double()
    want = z * torch.sigmoid(z)
    assert bool(((rows(o["x0"]) - want).abs() <= 64 * 2.0 ** -24 * (1 + z.abs()) + (u * want.abs() if u > 1e-6 else 0)).all())
    # the stack: rebuilt by the backward from its own output, to what the layers' inverse promises
    assert (rows(o["h"]) - rows(o["x0"])).abs().max() <= (1e-4 if dtype == torch.float32 else 0.25)
    # the head: loss and its gradients from the features that it was given
    y = m.plane()
    h = o["x0"].clone()
    for l in range(2):
        gsr.gsr_layer_forward(m.graph, m.cfg, m.w[l], h, workspace=m.ws)
    mean, rstd = torch.empty_like(o["mean1"]), torch.empty_like(o["rstd1"])
    m.norm(1, h, y, mean, rstd)
    assert torch.equal(y, o["g"]) and torch.equal(mean, o["mean1"]) and torch.equal(rstd, o["rstd1"])
    f, t = rows(y), m.targets.long()
    logits = f @ m.table.double().t() + m.bias.double()
    known = t >= 0
    want = torch.nn.functional.cross_entropy(logits[known], t[known])
    assert abs(o["loss"].item() - want.item()) <= 1e-5 * abs(want.item())           # sums of 64 terms of logits of up to 40: 1e-6 each
    dz = (torch.softmax(logits, 1) - torch.nn.functional.one_hot(t.clamp(min=0), m.types)) * known[:, None] / known.sum()
    for got, exact in ((o["dtable"].double(), dz.t() @ f), (o["dbias"].double(), dz.sum(0))):
        assert (got - exact).norm() <= (1e-5 if dtype == torch.float32 else 1e-2) * exact.norm()
    # the second norm's gradient, and the first's from what the codes stand for, given what the calls before them left
    df = (dz @ m.table.double()).to(dtype).reshape(m.n, m.c, -1).permute(1, 0, 2).contiguous()
    dh, ddx = m.plane(), m.plane()
    gsr.gsr_group_norm_grad(df, mean, rstd, dh, x=h, gamma=m.gamma[1], beta=m.beta[1], act=gsr.GSR_ACT_SILU, graph_ptr=m.ptr)
    for l in (1, 0):
        dw = torch.zeros_like(m.w[l])
        gsr.gsr_layer_backward(m.graph, m.cfg, m.w[l], h, dh, dw, workspace=m.ws)
        assert (dw - o[f"dw{l}"]).norm() <= (1e-4 if dtype == torch.float32 else 3e-2) * dw.norm()
    kept = m.plane()
    gsr.gsr_checkpoint_load(o["codes"], o["scales"], kept)
    assert (rows(kept) - x).abs().max() <= x.abs().max() / 254 * 1.01 + u * x.abs().max()
    if dtype == torch.float32:
        gsr.gsr_group_norm_grad(dh, o["mean0"], o["rstd0"], ddx, x=kept, gamma=m.gamma[0], beta=m.beta[0], act=gsr.GSR_ACT_SILU, graph_ptr=m.ptr)
        assert (rows(ddx) - rows(o["dx"])).norm() <= 1e-4 * rows(ddx).norm()
        dembed = torch.zeros((m.types, m.d), dtype=torch.float64, device=dev()).index_add_(0, m.ids.long(), rows(o["dx"]))
        assert (o["dembed"].double() - dembed).norm() <= 1e-5 * dembed.norm()


def test_gradient_of_a_whole_step_against_differences():
    """The loss along a direction of each parameter: to 2e-3 for the step's own curvature, and behind the first norm, whose input is kept in 8 bits (a value to
    1 / 254 of its block's largest, so to some 1e-2), to 5e-2."""
    m = Model(torch.float32, seed=3, k=32)             # every column kept: a selection has steps where its columns change
    o = m.buffers()
    m.step(o)
    grads = [(m.gamma[1], o["dgamma1"], 2e-3), (m.beta[1], o["dbeta1"], 2e-3), (m.bias, o["dbias"], 2e-3), (m.w[1], o["dw1"], 2e-3), (m.gamma[0], o["dgamma0"], 5e-2),
             (m.table, o["dtable"] + o["dembed"], 5e-2)]
    gen = torch.Generator(device="cuda").manual_seed(9)
    for p, g, tol in grads:
        v = g / g.norm() + 0.1 * torch.randn(p.shape, generator=gen, device=dev()) / p.numel() ** 0.5
        kept, losses = p.clone(), []
        h = 2e-3 / float(g.norm())          # moves the loss by 4e-3, thousands of its roundings
        for sign in (1, -1):
            p.copy_(kept + sign * h * v)
            q = m.buffers()
            m.step(q)
            losses.append(q["loss"].double().item())
        p.copy_(kept)
        slope, along = (losses[0] - losses[1]) / (2 * h), float((g.double() * v.double()).sum())
        assert abs(slope - along) <= tol * abs(along), (slope, along)


def test_a_step_captured_and_replayed():
    m = Model(torch.float32, seed=5)
    side = torch.cuda.Stream()
    got = m.buffers()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step(got)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step(got)
    for i in range(3):
        m.table.add_(0.1 * torch.randn_like(m.table))
        want = m.buffers()
        m.step(want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(got[k], want[k]), (i, k)
