"""The operators of a streaming block on tensors whose offsets pass 32 bits."""
import pytest
import torch

import test_linear_act as L
import test_rmsnorm as N
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
BF = dict(dtype=torch.bfloat16, device=DEV)


def filled(*shape, seed):
    """Normal numbers, without a tensor of four times the size in between."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.empty(*shape, **BF)
    flat = t.view(-1)
    step = 1 << 27
    for at in range(0, flat.numel(), step):
        flat[at:at + step] = torch.randn(min(step, flat.numel() - at), generator=g, device=DEV)
    return t


@pytest.mark.gpu
def test_rmsnorm_of_more_than_4_gib():
    rows, C = 1_700_000, 1280
    x = filled(rows, C, seed=1)
    y, s = torch.empty_like(x), torch.empty_like(x)
    gamma = torch.ones(C, device=DEV)
    B.dsattn_rmsnorm(rows, C, x, y, residual=x, gamma=gamma, sum_out=s)
    torch.cuda.synchronize()
    for at in (0, 1_677_700, rows - 40):  # (row 1,677,721 is the first one past 2^31 numbers)
        part = x[at:at + 40].cpu()
        N.check(40, C, "bf16", "bf16", part, part, gamma.cpu(), 1e-6, s[at:at + 40], y[at:at + 40], None)


@pytest.mark.gpu
@pytest.mark.parametrize("c_in,c_out,rows", [(320, 4096, 600_000), (4096, 320, 600_000)])
def test_linear_act_of_more_than_4_gib(c_in, c_out, rows):
    x, w = filled(rows, c_in, seed=2), filled(c_out, c_in, seed=3)
    r = filled(rows, c_out, seed=4)
    y = torch.empty(rows, c_out, **BF)
    B.dsattn_linear_act(rows, c_in, c_out, x, [w], y, residual=r, act=B.DSATTN_ACT_SILU)
    torch.cuda.synchronize()
    for at in (0, 524_200, rows - 300):
        t = {"X": x[at:at + 300], "W": [w], "sx": None, "sw": None, "b": None, "R": r[at:at + 300]}
        want, tol = L.reference(t, "silu", "bf16")
        assert ((y[at:at + 300].double() - want).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 3, 20, 80])
def test_sink_caches_of_more_than_4_gib(T):
    """2.3 billion numbers a cache: positions are the same as in a problem of their own."""
    P, h, D, sinks, window, ring = 3000, 8, 80, 4, 1100, 1200
    C, slots = h * D, sinks + ring
    Kc, Vc = filled(1, slots, P, C, seed=5), filled(1, slots, P, C, seed=6)
    q, k, v = (filled(1, T, P, C, seed=s) for s in (7, 8, 9))
    start = torch.full((1,), 5000, dtype=torch.int32, device=DEV)
    few = torch.tensor([0, 1, 1499, 2300, 2999], device=DEV)
    small = [t.index_select(2, few).contiguous() for t in (q, k, v, Kc, Vc)]

    def call(n, q, k, v, Kc, Vc):
        o = torch.zeros_like(q)
        space = torch.empty(B.dsattn_sink_workspace(1, T, n, h, h, D, sinks, window, ring), dtype=torch.uint8, device=DEV)
        B.dsattn_sink_forward(1, T, n, h, h, D, sinks, window, ring, q, k, v, o, Kcache=Kc, Vcache=Vc, start=start,
                              workspace=space)
        return o

    o = call(P, q, k, v, Kc, Vc)
    want = call(len(few), *small)
    torch.cuda.synchronize()
    # (few positions take another split of the frames: weights and output in bf16 either way, |v| to 6, means of 1,000)
    assert ((o.index_select(2, few).float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 6 * 2.0 ** -8 * 0.1).all()
    assert torch.equal(Kc.index_select(2, few), small[3]) and torch.equal(Vc.index_select(2, few), small[4])
