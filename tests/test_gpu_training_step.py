"""The operators as a training step uses them, together with the layers: flex-convolution, layer norm, class scores by a second
flex-convolution, log probabilities, all gradients, AdamW; against the float64 oracles, and captured into a graph."""
import numpy as np
import pytest
import torch

import oracle
import paper_1803_07289_amd as fx
from oracle import operators as ref
from gpu_util import TOL, dev, say
from helpers import rel_err
from workloads import CONFIGS, make_inputs

pytestmark = pytest.mark.gpu

CLASSES, WIDTH = 13, 64


def problem(layout):
    cfg = type(CONFIGS[0])(**{**CONFIGS[0].__dict__, "Din": 9, "Dout": WIDTH, "B": 2})
    x = make_inputs(cfg, n_override=600)
    rng = np.random.default_rng(12)
    f = lambda *shape: rng.standard_normal(shape).astype(np.float32)
    host = [x.theta, x.bias, 1 + 0.1 * f(WIDTH), 0.1 * f(WIDTH), f(3, WIDTH, CLASSES) / 30, f(WIDTH, CLASSES) / 30]
    target = rng.integers(0, CLASSES, (2, 600)).astype(np.int32)
    target[0, ::7] = -1
    lay = (lambda a: dev(a.transpose(0, 2, 1))) if layout == fx.BNC else dev
    return x, host, target, lay(x.feat)


class Step:
    def __init__(self, layout, bits):
        self.layout = layout
        self.x, self.host, self.target, self.feat = problem(layout)
        self.pos, self.nbr, self.t = dev(self.x.pos), dev(self.x.nbr), dev(self.target)
        self.params = [dev(p) for p in self.host]
        self.state = fx.flexadamw_state(self.params, bits)
        self.plan = fx.flexadamw_plan_build(self.params, *self.state, weight_decay=[0.1, 0.1, 0, 0, 0.1, 0.1])
        self.edges = fx.flex_inedges_build(self.nbr)
        n = int((self.target >= 0).sum())
        self.gl = torch.full(self.target.shape, -1.0 / n, device="cuda")
        self.gh = torch.full(self.target.shape, 0.05 / n, device="cuda")

    def __call__(self):
        theta, bias, w, b, theta2, bias2 = self.params
        L = self.layout
        h = fx.flexconv_fwd(self.feat, self.pos, self.nbr, theta, bias, layout=L)
        y, mean, rstd = fx.flexnorm_fwd(h, w, b, layout=L)
        scores = fx.flexconv_fwd(y, self.pos, self.nbr, theta2, bias2, layout=L)
        logp, ent, lse, _, best = fx.flexlogp_fwd(scores, self.t, top=1, layout=L)
        g = fx.flexlogp_bwd(scores, self.t, lse, ent, self.gl, self.gh, layout=L)
        g, gt2, gb2 = fx.flexconv_bwd(y, self.pos, self.nbr, theta2, bias2, g, layout=L, in_edges=self.edges)
        g, gw, gb = fx.flexnorm_bwd(h, w, g, mean, rstd, layout=L)
        _, gt, gbias = fx.flexconv_bwd(self.feat, self.pos, self.nbr, theta, bias, g, layout=L, in_edges=self.edges, need_feat=False)
        grads = [gt, gbias, gw, gb, gt2, gb2]
        fx.flexadamw_step(self.plan, grads, 1e-3)
        return logp, best, grads

    def reference(self):
        """(logp, gradients) in float64."""
        x, p = self.x, [np.asarray(v, np.float64) for v in self.host]
        rows = lambda a: a.transpose(0, 2, 1).reshape(-1, a.shape[1])
        back = lambda a: np.ascontiguousarray(a.reshape(2, 600, -1).transpose(0, 2, 1)).astype(np.float32)
        h = rows(oracle.flexconv_fwd(x.feat, x.pos, x.nbr, self.host[0], self.host[1]))
        y, mean, rstd = ref.norm_fwd(h, p[2], p[3])
        s = rows(oracle.flexconv_fwd(back(y), x.pos, x.nbr, self.host[4], self.host[5]))
        t = self.target.reshape(-1)
        logp, ent, lse, _, _ = ref.logp_fwd(s, t, 1)
        n = int((t >= 0).sum())
        g = ref.logp_bwd(s, t, lse, ent, np.full(t.size, -1.0 / n), np.full(t.size, 0.05 / n))
        g, gt2, gb2 = oracle.flexconv_bwd(back(y), x.pos, x.nbr, self.host[4], self.host[5], back(g))
        g, gw, gb = ref.norm_bwd(h, p[2], rows(np.asarray(g)), mean, rstd)
        _, gt, gbias = oracle.flexconv_bwd(x.feat, x.pos, x.nbr, self.host[0], self.host[1], back(g))
        return logp.reshape(2, 600), [gt, gbias, gw, gb, gt2, gb2]


@pytest.mark.parametrize("layout", [fx.BNC, fx.BCN], ids=["bnc", "bcn"])
def test_a_step_against_the_oracles(layout):
    say(f"training step {layout}")
    step = Step(layout, 32)
    before = [p.double().cpu().numpy() for p in step.params]
    logp, best, grads = step()
    want, wgrads = step.reference()
    # the layers' own tolerance, twice over for two of them one behind the other
    assert rel_err(logp.cpu().numpy(), want) <= 2 * TOL
    for got, w in zip(grads, wgrads):
        assert rel_err(got.cpu().numpy(), w) <= 4 * TOL
    for i, (p, g) in enumerate(zip(before, grads)):
        after, _, _ = ref.adamw(p, 0 * p, 0 * p, g.double().cpu().numpy(), 1, 1e-3, 0.9, 0.999, 1e-8, [0.1, 0.1, 0, 0, 0.1, 0.1][i])
        assert np.max(np.abs(step.params[i].double().cpu().numpy() - after)) <= 1e-3 * 2.0 ** -18 + 2.0 ** -22 * np.abs(p).max()


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_replay_from_a_graph(bits):
    """Forward, backward and update captured once; every replay is the eager run's next step."""
    a, b = Step(fx.BNC, bits), Step(fx.BNC, bits)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    a()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = b()
    for k in range(3):
        for t in (captured[0], captured[1], *captured[2]):
            t.fill_(7) if t.dtype == torch.int32 else t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        eager = a()                                                  # eager work between the replays
        torch.cuda.synchronize()
        for x, y in zip((captured[0], captured[1], *captured[2], *b.params), (eager[0], eager[1], *eager[2], *a.params)):
            assert torch.equal(x, y), f"replay {k}"
    assert a.plan.steps() == b.plan.steps() == 4


def test_two_streams_at_once_and_two_graphs():
    """Calls on two streams, each with scratch memory of its own, and two captured calls replayed one behind the other."""
    x = [torch.randn(1, 3001, 100, device="cuda") for _ in range(2)]
    big = [torch.randn(1, 2, 100_000, device="cuda") for _ in range(2)]
    w = torch.ones(100, device="cuda")

    def work(i):
        y, mean, rstd = fx.flexnorm_fwd(x[i], w, w, layout=fx.BNC)
        return fx.flexnorm_bwd(x[i], w, y, mean, rstd, layout=fx.BNC) + fx.flexlogp_fwd(big[i], top=20, layout=fx.BNC)[1:]
    want = [[t.clone() for t in work(i)] for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = work(i)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    kept = []
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            kept.append(work(i))
    for k in range(3):
        for i, g in enumerate(graphs):
            for t in kept[i]:
                t.zero_()
            g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(kept[i], want[i])), f"replay {k}"
        work(0)
        torch.cuda.synchronize()
