"""Tensors of more than 2^32 bytes and 2^31 numbers: what lies behind those borders against the same rows alone.  Rows in front are
zeros (or hold what the rows behind hold), so that sums over all rows are those of the last."""
import pytest
import torch

import test_layernorm as N
import test_linear_act_grad as G
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"


def tail(rows, C, n, seed):
    """A tensor of zeros but for its last n rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.zeros(rows, C, dtype=torch.bfloat16, device=DEV)
    t[-n:] = torch.randn(n, C, generator=g, device=DEV).bfloat16()
    return t


@pytest.mark.gpu
def test_layer_norm_and_its_gradients():
    rows, C, n = (1 << 31) // 1280 + 5000, 1280, 333
    x, dy = tail(rows, C, n, 1), tail(rows, C, n, 2)
    g = torch.Generator(device=DEV).manual_seed(3)
    gamma, beta = 1 + 0.1 * torch.randn(C, generator=g, device=DEV), torch.randn(C, generator=g, device=DEV)
    y = torch.empty_like(x)
    B.dsattn_layernorm(rows, C, x, y, gamma=gamma, beta=beta)
    torch.cuda.synchronize()
    N.check("bf16", "bf16", x[-n:].cpu(), None, gamma.cpu(), beta.cpu(), 1e-6, None, y[-n:])
    assert (y[:-n] == beta.bfloat16()).all()
    dg, db = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    ws = torch.empty(B.dsattn_layernorm_backward_workspace(rows, C), dtype=torch.uint8, device=DEV)
    B.dsattn_layernorm_backward(rows, C, x, dy, y, gamma=gamma, dgamma=dg, dbeta=db, workspace=ws)
    torch.cuda.synchronize()
    want = N.gradients(x[-n:].cpu(), None, gamma.cpu(), 1e-6, dy[-n:].cpu(), None)
    N.near(y[-n:].float(), want[0], N.half_step("bf16"))
    N.near(dg, want[1])
    N.near(db, want[2])
    assert (y[:-n] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("Bs,T,P,C", [(1, 40, 42000, 1280), (2, 1700000, 1, 640)])
def test_recurrence_and_its_gradients(Bs, T, P, C):
    """All streams, positions and frames hold a few patterns by turns: results repeat, or settle to what repeats."""
    g = torch.Generator(device=DEV).manual_seed(4)
    period = 50 if P == 1 else T
    x, gt, dy = (torch.empty(Bs, T, P, C, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    for t in (x, gt, dy):
        pattern = torch.randn(1, period, 1, C, generator=g, device=DEV).bfloat16()
        t.view(Bs, T // period, period, P, C).copy_(pattern.view(1, 1, period, 1, C).expand(Bs, T // period, period, P, C))
    n = 4 * period if P == 1 else T  # (gates of ordinary size forget in 200 frames)
    y, dx, dg = (torch.empty_like(x) for _ in range(3))
    S = torch.empty(Bs, -(-T // 16), P, C, device=DEV)
    ws = torch.empty(max(16, B.dsattn_gated_scan_workspace(Bs, T, P, C)), dtype=torch.uint8, device=DEV)
    end = torch.empty(Bs, P, C, device=DEV)
    B.dsattn_gated_scan(Bs, T, P, C, x, gt, y, end_state=end, states=S, workspace=ws)
    B.dsattn_gated_scan_backward(Bs, T, P, C, x, gt, S, dy, dx, dg, workspace=ws)
    torch.cuda.synchronize()
    # one stream and position of it, alone
    xs, gs, ds = (t[:1, :n, :1].contiguous() for t in (x, gt, dy))
    ys, dxs, dgs = (torch.empty_like(xs) for _ in range(3))
    Ss, es = torch.empty(1, -(-n // 16), 1, C, device=DEV), torch.empty(1, 1, C, device=DEV)
    w2 = torch.empty(max(16, B.dsattn_gated_scan_workspace(1, n, 1, C)), dtype=torch.uint8, device=DEV)
    B.dsattn_gated_scan(1, n, 1, C, xs, gs, ys, end_state=es, states=Ss, workspace=w2)
    B.dsattn_gated_scan_backward(1, n, 1, C, xs, gs, Ss, ds, dxs, dgs, workspace=w2)
    torch.cuda.synchronize()
    # the two differ in the order of 32-bit sums (a step of 16 bits then: 2^-7), and by what was forgotten
    def alike(a, b):
        return ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-4).all()

    if P > 1:
        for whole, one in ((y, ys), (dx, dxs), (dg, dgs)):
            assert alike(whole, one.expand_as(whole))
        assert alike(end, es.expand_as(end))
    else:
        mid = T // 2 // period * period  # (a multiple of the period, as n is)
        for at in (mid, T):
            assert alike(y[:, at - period:at], ys[:, n - period:].expand(Bs, -1, -1, -1))
        assert alike(end, es.expand_as(end))
        for at in (mid, 0):  # from a multiple of the period on
            keep = slice(at, at + period)
            assert alike(dx[:, keep], dxs[:, :period].expand(Bs, -1, -1, -1))
        assert alike(dg[:, mid:mid + period], dgs[:, 2 * period:3 * period].expand(Bs, -1, -1, -1))


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated,K,N_", [("none", False, 64, 1288), ("gelu", True, 640, 648), ("silu", False, 1288, 64)])
def test_gradients_of_a_product(act, gated, K, N_):
    widest = max(K, N_ * (2 if gated else 1))
    rows, n = (1 << 31) // widest + 3000, 700
    t = G.inputs(n, K, N_, "bf16", act, 6, gated, True)
    X, dY = (torch.zeros(rows, c, dtype=torch.bfloat16, device=DEV) for c in (K, N_))
    X[-n:], dY[-n:] = t["X"], t["dY"]
    big = dict(t, X=X, dY=dY)
    dX, dW, db = torch.empty_like(X), [torch.empty_like(w) for w in t["W"]], [torch.empty(N_, device=DEV) for _ in t["W"]]
    G.call(big, rows, K, N_, "bf16", act, dX, dW, db)
    torch.cuda.synchronize()
    rx, rw, rb = G.reference(t, act)
    G.near(dX[-n:], rx, "dX")
    for k in range(len(dW)):
        G.near(dW[k], rw[k], f"dW[{k}]")
        G.near(db[k], rb[k], f"dbias[{k}]")
    assert (dX[:-n] == 0).all()
