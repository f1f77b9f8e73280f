"""The operators of a recurrent block as they are used together, forward and backward: norm, projections of inputs and gates, recurrence,
output projection, norm with the residual's addition, gated feed-forward, the way back; then their gradients in the other order.

Each step is compared with its formula in 64 bits on the inputs that it really had, so that the tolerances are those of the
single operators (test_layernorm.py, test_linear_act.py, test_gated_scan.py, test_linear_act_grad.py)."""
import pytest
import torch

import test_gated_scan as R
import test_layernorm as N
import test_linear_act as L
import test_linear_act_grad as G
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
NONE, GELU = B.DSATTN_ACT_NONE, B.DSATTN_ACT_GELU


class Block:
    """One block's weights, state, buffers and gradients."""

    def __init__(self, Bs, T, P, C, hidden, dtype, seed, train=True):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype, self.dt, self.code = dtype, L.TORCH[dtype], L.CODE[dtype]
        self.Bs, self.T, self.P, self.C, self.hidden, self.rows = Bs, T, P, C, hidden, Bs * T * P
        self.shape = (Bs, T, P, C)

        def rand(*s):
            return torch.randn(*s, generator=g, device=DEV)

        self.w = {n: (rand(o, i) * i ** -0.5).to(self.dt) for n, o, i in (
            ("in", C, C), ("decay", C, C), ("out", C, C), ("gate", hidden, C), ("value", hidden, C), ("back", C, hidden))}
        self.b = {n: 0.1 * rand(w.shape[0]) + (2.0 if n == "decay" else 0.0) for n, w in self.w.items()}
        self.gamma, self.beta = [1 + 0.1 * rand(C) for _ in range(2)], [0.1 * rand(C) for _ in range(2)]
        self.h, self.hT = rand(Bs, P, C), torch.empty(Bs, P, C, device=DEV)

        def buf(c):
            return torch.empty(self.rows, c, device=DEV, dtype=self.dt)

        self.n1, self.x, self.g, self.s, self.x1, self.x2, self.n2, self.y = (buf(C) for _ in range(8))
        self.f = buf(hidden)
        self.states = torch.empty(Bs, -(-T // B.DSATTN_SCAN_FRAMES), P, C, device=DEV)
        need = [B.dsattn_gated_scan_workspace(Bs, T, P, C, io_dtype=self.code)]
        if train:
            self.df = buf(hidden)
            self.dn2, self.dx2, self.ds, self.dv, self.dg, self.dn1, self.dn1b, self.dx = (buf(C) for _ in range(8))
            self.dw, self.db = {n: torch.empty_like(w) for n, w in self.w.items()}, {n: torch.empty_like(b) for n, b in self.b.items()}
            self.dgamma, self.dbeta = ([torch.empty(C, device=DEV) for _ in range(2)] for _ in range(2))
            self.dh, self.dhT = torch.empty_like(self.h), rand(Bs, P, C)
            need.append(B.dsattn_layernorm_backward_workspace(self.rows, C, io_dtype=self.code))
            for names, act in ((["back"], NONE), (["gate", "value"], GELU), (["in"], NONE)):
                o, i = self.w[names[0]].shape
                need.append(B.dsattn_linear_act_backward_workspace(self.rows, i, o, n_w=len(names), act=act, io_dtype=self.code))
        # one workspace for all: calls on one stream follow each other
        self.space = torch.full((max(need + [16]),), 255, dtype=torch.uint8, device=DEV)

    def linear(self, x, names, y, act=NONE, residual=None):
        o, i = self.w[names[0]].shape
        B.dsattn_linear_act(self.rows, i, o, x, [self.w[n] for n in names], y, biases=[self.b[n] for n in names], residual=residual,
                            act=act, io_dtype=self.code)

    def linear_back(self, x, names, dy, dx, act=NONE):
        o, i = self.w[names[0]].shape
        B.dsattn_linear_act_backward(self.rows, i, o, x, [self.w[n] for n in names], dy, dX=dx, dWs=[self.dw[n] for n in names],
                                     dbiases=[self.db[n] for n in names], biases=[self.b[n] for n in names], act=act,
                                     workspace=self.space, io_dtype=self.code)

    def forward(self, x, h_in, h_out):
        B.dsattn_layernorm(self.rows, self.C, x, self.n1, gamma=self.gamma[0], beta=self.beta[0], io_dtype=self.code)
        self.linear(self.n1, ["in"], self.x)
        self.linear(self.n1, ["decay"], self.g)
        B.dsattn_gated_scan(*self.shape, self.x, self.g, self.s, mode=B.DSATTN_SCAN_NORM, start_state=h_in, end_state=h_out,
                            states=self.states, workspace=self.space, io_dtype=self.code)
        self.linear(self.s, ["out"], self.x1)
        B.dsattn_layernorm(self.rows, self.C, self.x1, self.n2, residual=x, gamma=self.gamma[1], beta=self.beta[1], sum_out=self.x2,
                           io_dtype=self.code)
        self.linear(self.n2, ["gate", "value"], self.f, act=GELU)
        self.linear(self.f, ["back"], self.y, residual=self.x2)

    def backward(self, x, dy):
        self.linear_back(self.f, ["back"], dy, self.df)
        self.linear_back(self.n2, ["gate", "value"], self.df, self.dn2, act=GELU)
        B.dsattn_layernorm_backward(self.rows, self.C, self.x1, self.dn2, self.dx2, residual=x, gamma=self.gamma[1], dsum=dy,
                                    dgamma=self.dgamma[1], dbeta=self.dbeta[1], workspace=self.space, io_dtype=self.code)
        self.linear_back(self.s, ["out"], self.dx2, self.ds)
        B.dsattn_gated_scan_backward(*self.shape, self.x, self.g, self.states, self.ds, self.dv, self.dg, mode=B.DSATTN_SCAN_NORM,
                                     dend_state=self.dhT, dstart_state=self.dh, workspace=self.space, io_dtype=self.code)
        self.linear_back(self.n1, ["in"], self.dv, self.dn1)
        self.linear_back(self.n1, ["decay"], self.dg, self.dn1b)
        self.dn1.add_(self.dn1b)
        B.dsattn_layernorm_backward(self.rows, self.C, x, self.dn1, self.dx, gamma=self.gamma[0], dsum=self.dx2,
                                    dgamma=self.dgamma[0], dbeta=self.dbeta[0], workspace=self.space, io_dtype=self.code)

    def results(self):
        return [self.y, self.hT, self.dx, self.dh, *self.dw.values(), *self.db.values(), *self.dgamma, *self.dbeta]

    # ---- each step against its formula
    def check_linear(self, x, names, y, act="none", residual=None):
        t = {"X": x, "W": [self.w[n] for n in names], "sx": None, "sw": None, "b": [self.b[n] for n in names], "R": residual}
        want, tol = L.reference(t, act, self.dtype)
        assert ((y.double() - want).abs() <= tol).all(), names

    def check_linear_back(self, x, names, dy, dx, act="none"):
        t = {"X": x, "W": [self.w[n] for n in names], "b": [self.b[n] for n in names], "dY": dy}
        rx, rw, rb = G.reference(t, act)
        G.near(dx, rx, names)
        for k, n in enumerate(names):
            G.near(self.dw[n], rw[k], n)
            G.near(self.db[n], rb[k], n)

    def check_norm_back(self, i, x, r, dy, ds, dx):
        want = N.gradients(x.cpu(), None if r is None else r.cpu(), self.gamma[i].cpu(), 1e-6, dy.cpu(), ds.cpu())
        N.near(dx.float(), want[0], N.half_step(self.dtype))
        N.near(self.dgamma[i], want[1])
        N.near(self.dbeta[i], want[2])

    def check(self, x, h_in, dy):
        N.check(self.dtype, self.dtype, x.cpu(), None, self.gamma[0].cpu(), self.beta[0].cpu(), 1e-6, None, self.n1)
        self.check_linear(self.n1, ["in"], self.x)
        self.check_linear(self.n1, ["decay"], self.g)
        xs, gs, ys, ds = (t.cpu().view(self.shape) for t in (self.x, self.g, self.s, self.ds))
        dv, dg = self.dv.cpu().view(self.shape), self.dg.cpu().view(self.shape)
        for b in range(self.Bs):
            h, e, _ = R.forward(xs[b], gs[b], h_in[b].cpu(), "norm", self.T)
            R.near(ys[b].float(), h[1:], e[1:], self.dtype, "s")
            R.near(self.hT[b], h[-1], e[-1], "f32", "state")
            rx, rg, r0 = R.backward(xs[b], gs[b], h_in[b].cpu(), "norm", self.T, ds[b], self.dhT[b].cpu())
            R.near(dv[b].float(), *rx, self.dtype, "dv")
            R.near(dg[b].float(), *rg, self.dtype, "dg")
            R.near(self.dh[b], *r0, "f32", "dh")
        self.check_linear(self.s, ["out"], self.x1)
        N.check(self.dtype, self.dtype, self.x1.cpu(), x.cpu(), self.gamma[1].cpu(), self.beta[1].cpu(), 1e-6, self.x2, self.n2)
        self.check_linear(self.n2, ["gate", "value"], self.f, "gelu")
        self.check_linear(self.f, ["back"], self.y, residual=self.x2)
        self.check_linear_back(self.f, ["back"], dy, self.df)
        self.check_linear_back(self.n2, ["gate", "value"], self.df, self.dn2, "gelu")
        self.check_norm_back(1, self.x1, x, self.dn2, dy, self.dx2)
        self.check_linear_back(self.s, ["out"], self.dx2, self.ds)
        self.check_linear_back(self.n1, ["decay"], self.dg, self.dn1b)
        self.check_norm_back(0, x, None, self.dn1, self.dx2, self.dx)


SHAPES = [(1, 3, 40, 320, 640), (2, 17, 9, 160, 328), (1, 24, 135, 320, 1280), (2, 300, 1, 128, 512), (3, 50, 1, 40, 72)]


def batches(blk, seed, n):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [[torch.randn(blk.rows, blk.C, generator=g, device=DEV).to(blk.dt) for _ in range(2)] for _ in range(n)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Bs,T,P,C,hidden", SHAPES)
def test_a_block_forward_and_backward(Bs, T, P, C, hidden, dtype):
    blk = Block(Bs, T, P, C, hidden, dtype, 1)
    for x, dy in batches(blk, 2, 2):
        blk.forward(x, blk.h, blk.hT)
        blk.backward(x, dy)
        torch.cuda.synchronize()
        blk.check(x, blk.h, dy)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Bs,T,P,C,hidden", SHAPES[1:4])
def test_a_captured_training_step_replays(Bs, T, P, C, hidden, dtype):
    """One graph with forward and backward pass, replayed with new inputs and eager work between; two blocks' graphs by turns."""
    eager = [Block(Bs, T, P, C, hidden, dtype, s) for s in (1, 2)]
    graphed = [Block(Bs, T, P, C, hidden, dtype, s) for s in (1, 2)]
    x_in, dy_in = batches(eager[0], 3, 1)[0]
    graphs = []
    for blk in graphed:
        blk.forward(x_in, blk.h, blk.hT)  # (kernels are loaded outside of the capture)
        blk.backward(x_in, dy_in)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            blk.forward(x_in, blk.h, blk.hT)
            blk.backward(x_in, dy_in)
        graphs.append(graph)
    for i, (x, dy) in enumerate(batches(eager[0], 4, 5)):
        for blk, graph, ref in zip(graphed, graphs, eager):
            x_in.copy_(x)
            dy_in.copy_(dy)
            blk.space.fill_(255)
            graph.replay()
            if i % 2:
                torch.cuda.synchronize()
            ref.forward(x, ref.h, ref.hT)
            ref.backward(x, dy)
            torch.cuda.synchronize()
            for a, b in zip(blk.results(), ref.results()):
                assert torch.equal(a, b), i


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P,C,hidden", [(40, 320, 640), (1, 128, 520)])
def test_a_stream_frame_by_frame_from_a_graph(P, C, hidden, dtype):
    """A graph of one frame, the state moved on in its place, against all frames in one call: the recurrence of few frames does the
    same arithmetic in both, and so do rows of every other operator that are as many (each frame alone in the eager block)."""
    T = 12
    blk, ref = Block(1, 1, P, C, hidden, dtype, 5, train=False), Block(1, 1, P, C, hidden, dtype, 5, train=False)
    x_in = torch.zeros(P, C, device=DEV, dtype=blk.dt)
    state = blk.h.clone()
    blk.forward(x_in, state, state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blk.forward(x_in, state, state)
    state.copy_(blk.h)
    h = ref.h.clone()
    xs, gs, ss = [], [], []
    for x, _ in batches(blk, 6, T):
        x_in.copy_(x)
        graph.replay()
        ref.forward(x, h, ref.hT)
        h.copy_(ref.hT)
        torch.cuda.synchronize()
        assert torch.equal(blk.y, ref.y) and torch.equal(state, h)
        xs.append(blk.x.clone())
        gs.append(blk.g.clone())
        ss.append(blk.s.clone())
    y, end = torch.empty(1, T, P, C, device=DEV, dtype=blk.dt), torch.empty_like(h)
    B.dsattn_gated_scan(1, T, P, C, torch.stack(xs), torch.stack(gs), y, mode=B.DSATTN_SCAN_NORM, start_state=ref.h, end_state=end,
                        io_dtype=blk.code)
    torch.cuda.synchronize()
    assert torch.equal(y[0], torch.stack(ss)) and torch.equal(end, h)


@pytest.mark.gpu
@pytest.mark.parametrize("Bs,T,P,C,hidden", [SHAPES[1], SHAPES[3]])
def test_two_streams_at_once(Bs, T, P, C, hidden):
    """Two blocks with buffers and workspaces of their own, on two streams, nothing waiting between their calls."""
    both, alone = ([Block(Bs, T, P, C, hidden, "bf16", s) for s in (1, 2)] for _ in range(2))
    data = batches(both[0], 7, 6)
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for x, dy in data:
        for blk, st in zip(both, streams):
            with torch.cuda.stream(st):
                blk.forward(x, blk.h, blk.hT)
                blk.backward(x, dy)
    for st in streams:
        st.synchronize()
    for blk, ref in zip(both, alone):
        for x, dy in data:
            ref.forward(x, ref.h, ref.hT)
            ref.backward(x, dy)
        torch.cuda.synchronize()
        for a, b in zip(blk.results(), ref.results()):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_calls_run_on_the_stream_they_are_given():
    blk, ref = (Block(1, 3, 40, 320, 640, "bf16", 3) for _ in range(2))
    x, dy = batches(blk, 8, 1)[0]
    ref.forward(x, ref.h, ref.hT)
    ref.backward(x, dy)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    rows, C = blk.rows, blk.C
    B.dsattn_layernorm(rows, C, x, blk.n1, gamma=blk.gamma[0], beta=blk.beta[0], stream=side)
    B.dsattn_gated_scan(*blk.shape, ref.x, ref.g, blk.s, mode=B.DSATTN_SCAN_NORM, start_state=blk.h, end_state=blk.hT,
                        workspace=blk.space, stream=side)
    B.dsattn_gated_scan_backward(*blk.shape, ref.x, ref.g, ref.states, ref.ds, blk.dv, blk.dg, mode=B.DSATTN_SCAN_NORM,
                                 dend_state=ref.dhT, dstart_state=blk.dh, workspace=blk.space, stream=side)
    B.dsattn_linear_act_backward(rows, C, 640, ref.n2, [ref.w["gate"], ref.w["value"]], ref.df, dX=blk.dn2,
                                 dWs=[blk.dw["gate"], blk.dw["value"]], dbiases=[blk.db["gate"], blk.db["value"]],
                                 biases=[ref.b["gate"], ref.b["value"]], act=GELU, workspace=blk.space, stream=side)
    B.dsattn_layernorm_backward(rows, C, ref.x1, ref.dn2, blk.dx2, residual=x, gamma=ref.gamma[1], dsum=dy, dgamma=blk.dgamma[1],
                                dbeta=blk.dbeta[1], workspace=blk.space, stream=side)
    side.synchronize()
    for name in ("n1", "s", "hT", "dv", "dg", "dh", "dn2", "dx2"):
        assert torch.equal(getattr(blk, name), getattr(ref, name)), name
    for n in ("gate", "value"):
        assert torch.equal(blk.dw[n], ref.dw[n]) and torch.equal(blk.db[n], ref.db[n])
    assert torch.equal(blk.dgamma[1], ref.dgamma[1]) and torch.equal(blk.dbeta[1], ref.dbeta[1])
