"""Frames that begin anew: a gate whose logit is minus infinity, or below -87, keeps nothing of the state before it or of the
gradient behind it, however large they are.  Then h_t = w(0) x_t with w(0) = 1 in every mode, 8 u off at most, and D_t
passes nothing on: what is in front of such a frame gives the bits that it gives alone."""
import pytest
import torch

import test_gated_scan as R
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
RESETS = {"f32": [float("-inf"), -3.4e38, -1000.0, -211.0, -120.0, -88.0], "bf16": [float("-inf"), -3.38e38, -1000.0, -88.0]}


def forward(shape, x, g, h0, mode, dtype, states):
    Y, hT = torch.empty_like(x), torch.empty_like(h0)
    B.dsattn_gated_scan(*shape, x, g, Y, mode=R.MODES[mode], start_state=h0, end_state=hT, states=states,
                        workspace=R.space(*shape, dtype), io_dtype=R.CODE[dtype])
    return Y, hT


@pytest.mark.gpu
@pytest.mark.parametrize("mode", list(R.MODES))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,P,C,at", [(1, 3, 40, 0), (40, 3, 40, 0), (40, 3, 40, 21), (600, 1, 64, 333), (600, 1, 64, 599), (35, 1, 1 << 16, 17),
                                      (35, 1, 1 << 18, 17)])
def test_nothing_is_kept_of_what_was_before(T, P, C, at, dtype, mode):
    shape = (1, T, P, C)
    for far in RESETS[dtype]:
        x, g, h0, dy, dend = (t.to(DEV) for t in R.inputs(*shape, dtype, 5))
        g[:, at] = far
        if at:  # a state of 1e38 in front of it
            x[:, at - 1], g[:, at - 1] = 1e38, -5.0
        h0, other = torch.full_like(h0, 1e38), torch.full_like(h0, -3e38)
        S = torch.empty(1, -(-T // R.STEP), P, C, device=DEV)
        Y, hT = forward(shape, x, g, h0, mode, dtype, S)
        torch.cuda.synchronize()
        xt = x[:, at].double()
        half = torch.finfo(R.TORCH[dtype]).eps / 2 if dtype == "bf16" else 0
        assert ((Y[:, at].double() - xt).abs() <= xt.abs() * (12 * R.U + half * (1 + 12 * R.U))).all()
        # another past gives the same states from there on
        x2 = x.clone()
        x2[:, :at] = -x2[:, :at]
        Y2, hT2 = forward(shape, x2, g, other, mode, dtype, None)
        assert torch.equal(Y2[:, at:], Y[:, at:]) and torch.equal(hT2, hT)
        # and no gradient comes through from behind: those of 1e30 are as those of 0
        out = []
        for big in (0.0, 1e30):
            dy2 = dy.clone()
            dy2[:, at:] = big
            dX, dG, dh = torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
            B.dsattn_gated_scan_backward(*shape, x, g, S, dy2, dX, dG, mode=R.MODES[mode], dend_state=torch.full_like(h0, big),
                                         dstart_state=dh, workspace=R.space(*shape, dtype), io_dtype=R.CODE[dtype])
            torch.cuda.synchronize()
            assert (dG[:, at] == 0).all()
            out.append((dX[:, :at], dG[:, :at], dh))
        assert all(torch.equal(a, b) for a, b in zip(*out))
        if not at:
            assert (out[0][2] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("mode", list(R.MODES))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_gate_that_is_not_a_number_is_not_a_reset(dtype, mode):
    T, C = 40, 64
    x, g, h0, _, _ = (t.to(DEV) for t in R.inputs(1, T, 1, C, dtype, 6))
    g[:, 20, :, 7] = float("nan")
    Y, hT = forward((1, T, 1, C), x, g, h0, mode, dtype, None)
    torch.cuda.synchronize()
    assert Y[0, 20:, 0, 7].isnan().all() and hT[0, 0, 7].isnan()
    keep = [c for c in range(C) if c != 7]
    assert Y[..., keep].isfinite().all() and Y[0, :20].isfinite().all()
