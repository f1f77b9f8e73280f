"""The operators of a streaming transformer block as they are used together: norm, projections, attention over the
cache, output projection with the residual, norm with the residual's addition, gated feed-forward and the way back.

Each step is compared with its formula in 64 bits on the inputs that it really had (the step before's outputs),
so that the tolerances are those of the single operators (test_rmsnorm.py, test_linear_act.py, test_sink_attn.py)."""
import pytest
import torch

import test_linear_act as L
import test_rmsnorm as N
import test_sink_attn as S
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"


class Block:
    """One block's weights, cache and buffers; 8-bit products where `eight`."""

    def __init__(self, T, P, heads, kv_heads, D, sinks, window, hidden, eight, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def rand(*s):
            return torch.randn(*s, generator=g, device=DEV)

        self.T, self.P, self.h, self.hk, self.D, self.sinks, self.window = T, P, heads, kv_heads, D, sinks, window
        self.C, self.Ckv, self.hidden, self.eight = heads * D, kv_heads * D, hidden, eight
        self.ring, self.rows, C = window + T - 1, T * P, heads * D
        self.dt = "e4m3" if eight else "bf16"
        self.w, self.sw = {}, {}
        for name, n, k in (("q", C, C), ("k", self.Ckv, C), ("v", self.Ckv, C), ("o", C, C), ("gate", hidden, C),
                           ("value", hidden, C), ("back", C, hidden)):
            w = rand(n, k) * k ** -0.5
            if eight and name not in ("o", "back"):
                s = w.abs().amax(1) / 448
                self.w[name], self.sw[name] = (w / s[:, None]).to(torch.float8_e4m3fn), s
            else:
                self.w[name] = w.bfloat16()
        self.bias = {n: 0.1 * rand(w.shape[0]) for n, w in self.w.items()}
        self.gamma = [1 + 0.1 * rand(C) for _ in range(2)]
        bf = dict(dtype=torch.bfloat16, device=DEV)
        self.n = torch.empty(self.rows, C, device=DEV, dtype=L.TORCH[self.dt])
        self.n2, self.sn = torch.empty_like(self.n), [torch.empty(self.rows, device=DEV) for _ in range(2)]
        self.q, self.a, self.x1, self.x2 = (torch.empty(self.rows, C, **bf) for _ in range(4))
        self.k, self.v = (torch.empty(self.rows, self.Ckv, **bf) for _ in range(2))
        self.f = torch.empty(self.rows, hidden, **bf)
        self.y = torch.empty(self.rows, C, **bf)
        self.Kc, self.Vc = (torch.full((1, sinks + self.ring, P, self.Ckv), float("nan"), **bf) for _ in range(2))
        self.start = torch.zeros(1, dtype=torch.int32, device=DEV)
        space = B.dsattn_sink_workspace(1, T, P, heads, kv_heads, D, sinks, window, self.ring)
        self.space = torch.empty(space, dtype=torch.uint8, device=DEV)

    def linear(self, x, sx, names, y, act=B.DSATTN_ACT_NONE, residual=None):
        w = [self.w[n] for n in names]
        eight = w[0].dtype == torch.float8_e4m3fn
        B.dsattn_linear_act(self.rows, w[0].shape[1], w[0].shape[0], x, w, y, biases=[self.bias[n] for n in names],
                            residual=residual, x_scales=sx if eight else None,
                            w_scales=[self.sw[n] for n in names] if eight else None, act=act,
                            io_dtype=B.DSATTN_E4M3 if eight else B.DSATTN_BF16, out_dtype=B.DSATTN_BF16)

    def norm(self, i, x, y, residual=None, total=None):
        B.dsattn_rmsnorm(self.rows, self.C, x, y, residual=residual, gamma=self.gamma[i], sum_out=total,
                         scales=self.sn[i] if self.eight else None,
                         out_dtype=B.DSATTN_E4M3 if self.eight else B.DSATTN_BF16)

    def step(self, x):
        """T new frames through the block; the stream's position moves on on the device."""
        self.norm(0, x, self.n)
        for name, y in (("q", self.q), ("k", self.k), ("v", self.v)):
            self.linear(self.n, self.sn[0], [name], y)
        B.dsattn_sink_forward(1, self.T, self.P, self.h, self.hk, self.D, self.sinks, self.window, self.ring, self.q,
                              self.k, self.v, self.a, Kcache=self.Kc, Vcache=self.Vc, start=self.start,
                              workspace=self.space)
        self.linear(self.a, None, ["o"], self.x1)
        self.norm(1, self.x1, self.n2, residual=x, total=self.x2)
        self.linear(self.n2, self.sn[1], ["gate", "value"], self.f, act=B.DSATTN_ACT_GELU)
        self.linear(self.f, None, ["back"], self.y, residual=self.x2)
        self.start.add_(self.T)

    # ---- each step against its formula
    def check_linear(self, x, sx, names, y, act="none", residual=None):
        eight = self.w[names[0]].dtype == torch.float8_e4m3fn
        t = {"X": x, "W": [self.w[n] for n in names], "sx": sx if eight else None,
             "sw": [self.sw[n] for n in names] if eight else None, "b": [self.bias[n] for n in names], "R": residual}
        want, tol = L.reference(t, act, "bf16")
        assert ((y.double() - want).abs() <= tol).all(), names

    def check_norm(self, i, x, y, residual=None, total=None):
        N.check(self.rows, self.C, "bf16", self.dt, x.cpu(), None if residual is None else residual.cpu(),
                self.gamma[i].cpu(), 1e-6, total, y, self.sn[i] if self.eight else None)

    def check(self, x, history, first):
        self.check_norm(0, x, self.n)
        for name, y in (("q", self.q), ("k", self.k), ("v", self.v)):
            self.check_linear(self.n, self.sn[0], [name], y)
        s = S.Stream(S.case("bf16", T=self.T, P=self.P, h=self.h, hk=self.hk, D=self.D, sinks=self.sinks,
                            window=self.window, ring=self.ring), 0)
        shape = (1, self.T, self.P, -1)
        s.start, s.Q, s.K, s.V = [first], *(t.cpu().view(*shape) for t in (self.q, self.k, self.v))
        s.Kc, s.Vc = history
        want, tol = s.reference(self.D ** -0.5)
        assert ((self.a.cpu().double().view_as(want) - want).abs() <= tol).all(), "attention"
        Kw, Vw = s.caches()
        assert S.same_bits(self.Kc, Kw) and S.same_bits(self.Vc, Vw)
        self.check_linear(self.a, None, ["o"], self.x1)
        self.check_norm(1, self.x1, self.n2, residual=x, total=self.x2)
        self.check_linear(self.n2, self.sn[1], ["gate", "value"], self.f, "gelu")
        self.check_linear(self.f, None, ["back"], self.y, residual=self.x2)


SHAPES = [(1, 40, 4, 4, 40, 2, 5, 320), (1, 160, 8, 8, 80, 4, 12, 1280), (3, 20, 8, 2, 64, 1, 7, 512), (24, 15, 5, 5, 64, 4, 16, 640),
          (7, 1, 8, 2, 128, 4, 30, 1024)]


def frames(blk, seed, steps):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [torch.randn(blk.rows, blk.C, generator=g, device=DEV).bfloat16() for _ in range(steps)]


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("T,P,h,hk,D,sinks,window,hidden", SHAPES)
def test_a_block_over_a_stream(T, P, h, hk, D, sinks, window, hidden, eight):
    blk = Block(T, P, h, hk, D, sinks, window, hidden, eight, 1)
    for i, x in enumerate(frames(blk, 2, 2 + 2 * window // T if T < 8 else 3)):
        history = blk.Kc.cpu(), blk.Vc.cpu()
        blk.step(x)
        torch.cuda.synchronize()
        blk.check(x, history, i * T)


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("T,P,h,hk,D,sinks,window,hidden", [SHAPES[1], SHAPES[2], (1, 1, 8, 2, 128, 4, 3000, 512)])
def test_a_captured_block_replays_every_frame(T, P, h, hk, D, sinks, window, hidden, eight):
    """One graph, replayed for every frame, with eager work between; and two blocks' graphs by turns."""
    steps = 12
    eager = [Block(T, P, h, hk, D, sinks, window, hidden, eight, s) for s in (1, 2)]
    graphed = [Block(T, P, h, hk, D, sinks, window, hidden, eight, s) for s in (1, 2)]
    xs = frames(eager[0], 5, steps)
    x_in = torch.empty_like(xs[0])
    graphs = []
    for blk in graphed:
        x_in.copy_(xs[0])
        blk.step(x_in)  # (kernels are loaded outside of the capture)
        blk.start.zero_()
        blk.Kc.fill_(float("nan"))
        blk.Vc.fill_(float("nan"))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            blk.step(x_in)
        graphs.append(graph)
    for i in range(steps):
        for blk, graph, ref in zip(graphed, graphs, eager):
            x_in.copy_(xs[i])
            graph.replay()
            if i % 2:
                torch.cuda.synchronize()
            ref.step(xs[i])
            torch.cuda.synchronize()
            for name in ("y", "a", "f", "Kc", "Vc"):
                assert S.same_bits(getattr(blk, name), getattr(ref, name)), (i, name)
            assert blk.start.item() == ref.start.item() == (i + 1) * T


@pytest.mark.gpu
def test_calls_run_on_the_stream_they_are_given():
    """A block on a side stream, by the stream argument and by torch's current stream."""
    a, b = (Block(2, 40, 8, 8, 40, 2, 9, 640, False, 3) for _ in range(2))
    xs = frames(a, 7, 4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for x in xs:
            a.step(x)
    side.synchronize()
    for x in xs:
        b.step(x)
    torch.cuda.synchronize()
    assert S.same_bits(a.y, b.y) and S.same_bits(a.Kc, b.Kc)
    x, y = xs[0], torch.zeros_like(xs[0])
    s2 = torch.cuda.Stream()
    s2.wait_stream(torch.cuda.current_stream())
    B.dsattn_rmsnorm(a.rows, a.C, x, y, gamma=a.gamma[0], stream=s2)
    B.dsattn_linear_act(a.rows, a.C, a.C, y, [a.w["q"]], a.q, stream=s2)
    s2.synchronize()
    N.check(a.rows, a.C, "bf16", "bf16", x.cpu(), None, a.gamma[0].cpu(), 1e-6, None, y, None)
    t = {"X": y, "W": [a.w["q"]], "sx": None, "sw": None, "b": None, "R": None}
    want, tol = L.reference(t, "none", "bf16")
    assert ((a.q.double() - want).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,P,h,hk,D,sinks,window,hidden", [SHAPES[1], SHAPES[3], (1, 1, 8, 2, 128, 4, 3000, 512)])
def test_two_streams_at_once(T, P, h, hk, D, sinks, window, hidden):
    """Two blocks with buffers and workspaces of their own, on two streams, nothing waiting between their calls."""
    both = [Block(T, P, h, hk, D, sinks, window, hidden, True, s) for s in (1, 2)]
    alone = [Block(T, P, h, hk, D, sinks, window, hidden, True, s) for s in (1, 2)]
    xs = frames(both[0], 9, 10)
    side = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for x in xs:
        for blk, s in zip(both, side):
            with torch.cuda.stream(s):
                blk.step(x)
    torch.cuda.synchronize()
    for blk, ref in zip(both, alone):
        for x in xs:
            ref.step(x)
        torch.cuda.synchronize()
        for name in ("y", "a", "f", "Kc", "Vc"):
            assert S.same_bits(getattr(blk, name), getattr(ref, name)), name
