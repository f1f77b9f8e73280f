"""The gradients of a recurrent block that its own test goes past: those of the inputs' projection, whose dX is added to another's."""
import pytest
import torch

import test_linear_act_grad as G
import test_train_block as T


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Bs,T_,P,C,hidden", T.SHAPES)
def test_the_projection_of_the_inputs(Bs, T_, P, C, hidden, dtype):
    """dW and dbias against the formula, dX through its sum with the gates' (one rounding more, of the sum)."""
    blk = T.Block(Bs, T_, P, C, hidden, dtype, 1)
    (x, dy), = T.batches(blk, 2, 1)
    blk.forward(x, blk.h, blk.hT)
    blk.backward(x, dy)
    torch.cuda.synchronize()
    rx, rw, rb = G.reference({"X": blk.n1, "W": [blk.w["in"]], "b": [blk.b["in"]], "dY": blk.dv}, "none")
    G.near(blk.dw["in"], rw[0], "dW")
    G.near(blk.db["in"], rb[0], "dbias")
    half, both = torch.finfo(blk.dt).eps / 2, rx[0] + blk.dn1b.double()
    G.near(blk.dn1, (both, rx[1] * (1 + half) + half * both.abs()), "dX")
