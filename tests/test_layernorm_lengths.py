"""dsattn_layernorm and its backward pass at lengths that each go to a kernel of their own: lanes of a row by pieces of a lane, rows that
are whole pieces of 16 bytes and rows that are not, in both types and 8 bits; the sums of extreme rows; what lies behind a workspace."""
import pytest
import torch

import test_layernorm as N
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
# pieces of 4 (fp32) or 8 (bf16) numbers: up to 8, 16, 32, 64 x 1 to 4, 256 x 2 to 4, 1,024 x 2 (512 x 3 and 4 in the backward pass)
LENGTHS = [9, 30, 45, 56, 101, 104, 180, 201, 301, 304, 500, 501, 620, 700, 701, 800, 801, 1001, 1200, 1600, 1601, 2001, 2500, 2501, 3500,
           3501, 4500, 4501, 5000, 5001, 6000, 6001, 7000, 7001, 8191, 9001, 10000, 10001, 14000, 14001, 16381]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("C", LENGTHS)
def test_lengths(C, dtype, out):
    N.run(37, C, dtype, out, 500 + C)
    N.run(3, C, dtype, out, 501 + C, residual=False, affine=False, want_sum=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", LENGTHS)
def test_gradients(C, dtype):
    N.run_back(37, C, dtype, 600 + C)
    N.run_back(3, C, dtype, 601 + C, residual=False, affine=False, dsum=False)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [40, 1279, 1280, 5001, 20000])
def test_sums_of_rows_beyond_the_range_of_their_squares(C):
    """Rows of 2^-60, 2^-110, 2^90 and 2^120 times an ordinary one have its n, eps 0, and so its dgamma.  A number of the second may be
    below 2^-126 and is off by half of 2^-149 then, 2^-40 of the largest: that much in units of the deviation more in its n."""
    x, _, gamma, _, dy, _ = N.inputs(1, C, "f32", 6, False)
    x = x / x.abs().max()
    power = torch.tensor([1.0, 2.0 ** -60, 2.0 ** -110, 2.0 ** 90, 2.0 ** 120])
    dys = dy * torch.tensor([1.0, -0.5, 2.0, 0.25, 1.5])[:, None]
    dX, dg, db = torch.empty(5, C, device=DEV), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    B.dsattn_layernorm_backward(5, C, (x * power[:, None]).to(DEV), dys.to(DEV), dX, gamma=gamma.to(DEV), dgamma=dg, dbeta=db,
                                workspace=N.space(5, C, "f32"), io_dtype=B.DSATTN_F32, eps=0.0)
    torch.cuda.synchronize()
    _, want_g, want_b = N.gradients(x.expand(5, C), None, gamma, 0.0, dys, None)
    rstd = N.normed(x, None, 0.0)[3].item()
    N.near(dg, (want_g[0], want_g[1] + dys[2].double().abs() * 2.0 ** -40 * rstd))
    N.near(db, want_b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", [(1, 1), (3, 7), (8, 1280), (9, 320), (64, 640), (300, 1279), (2000, 320), (5000, 24), (2100, 4096), (3, 16384),
                                    (130, 20000)])
def test_nothing_behind_the_workspace_is_written(rows, C, dtype):
    need = B.dsattn_layernorm_backward_workspace(rows, C, io_dtype=N.CODE[dtype])
    x, r, gamma, _, dy, ds = (t.to(DEV) for t in N.inputs(rows, C, dtype, 3, True))
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    outs = []
    for ws in (room[:need], N.space(rows, C, dtype)):
        out = torch.empty_like(x), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
        B.dsattn_layernorm_backward(rows, C, x, dy, out[0], residual=r, gamma=gamma, dsum=ds, dgamma=out[1], dbeta=out[2], workspace=ws,
                                    io_dtype=N.CODE[dtype])
        torch.cuda.synchronize()
        outs.append(out)
    assert (room[need:] == 0xA5).all()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
