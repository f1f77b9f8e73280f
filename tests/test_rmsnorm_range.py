"""dsattn_rmsnorm of rows whose squares leave fp32's range, at either end.

Tolerances are those of test_rmsnorm.py: a factor of a power of two on a row is exact, so that the sum of squares has
the same relative error at every size.  (Every number here is at least 2^-20 of its row's norm or zero: what a
factor for the largest rows pushes below 2^-126 is not among them.)"""
import pytest
import torch

import test_rmsnorm as N
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
# powers of two that a row's numbers are multiplied with: squares of the first ones are zero in fp32, of the next
# ones subnormal, of the last ones infinite
SMALL, LARGE = [-120, -100, -76, -75, -74, -70, -64, -62, -50, -40], [55, 62, 64, 65, 100, 120]


def rows_of(C, dtype, powers, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(len(powers), C, generator=g)
    x = torch.where(x.abs() < 2.0 ** -6, 0.5, x) * 2.0 ** torch.tensor(powers, dtype=torch.float32)[:, None]
    return x.to(N.TORCH[dtype])


def run(x, r, gamma, dtype, out, eps):
    rows, C = x.shape
    S = torch.full((rows, C), float("nan"), device=DEV).to(N.TORCH[dtype])
    Y = torch.full((rows, C), float("nan"), device=DEV).to(N.TORCH[out])
    scales = torch.full((rows,), float("nan"), device=DEV) if out == "e4m3" else None
    B.dsattn_rmsnorm(rows, C, x.to(DEV), Y, residual=None if r is None else r.to(DEV), gamma=gamma.to(DEV), sum_out=S,
                     scales=scales, io_dtype=N.CODE[dtype], out_dtype=N.CODE[out], eps=eps)
    torch.cuda.synchronize()
    N.check(rows, C, dtype, out, x, r, gamma, eps, S, Y, scales)


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30, 1e-22, 1e-6])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("C", [1, 7, 40, 130, 320, 1280, 1866, 9999, 20000, 65536])
def test_rows_of_every_size(C, dtype, out, eps):
    """Rows of every size among each other (a wavefront has up to eight), with eps below, near and above their squares."""
    powers = [0] + SMALL + [3] + LARGE + [-1]
    print(f"[case] rmsnorm of rows of every size, {C} {dtype} -> {out}, eps {eps}", flush=True)
    gamma = 1.0 + 0.3 * torch.rand(C, generator=torch.Generator().manual_seed(C))
    run(rows_of(C, dtype, powers, C), None, gamma, dtype, out, eps)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("C", [40, 1280, 20000])
def test_with_a_residual_of_the_same_size(C, dtype, out):
    powers = SMALL + LARGE
    x = rows_of(C, dtype, powers, C + 1)
    r = rows_of(C, dtype, powers, C + 2).abs() * x.sign()  # (no sum is smaller than its operands)
    run(x, r, torch.ones(C), dtype, out, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [8, 320, 2560, 65536])
def test_subnormal_rows_in_place(C):
    """fp32 rows of subnormal numbers, and the largest ones, sum over the residual and output over the input."""
    x = torch.cat([rows_of(C, "f32", [-140], 3), rows_of(C, "f32", [124], 4), rows_of(C, "f32", [0], 5)])
    dx, dr = x.to(DEV), torch.zeros_like(x).to(DEV)
    gamma = torch.ones(C)
    B.dsattn_rmsnorm(3, C, dx, dx, residual=dr, gamma=gamma.to(DEV), sum_out=dr, io_dtype=B.DSATTN_F32, eps=0.0)
    torch.cuda.synchronize()
    assert torch.equal(dr.cpu(), x)
    N.check(3, C, "f32", "f32", x, torch.zeros_like(x), gamma, 0.0, dr, dx, None)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [24, 1280, 20000, 65536])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_nan_and_zeros_without_an_eps(C, dtype):
    """0 / 0 and infinity / infinity are no numbers, the rest of an infinite row is zero, rows beside them are as ever."""
    x = rows_of(C, dtype, [0, -100, 0, 100, 0, 0], 6)
    x[0], x[2, C // 2], x[4, C - 1] = 0, float("-inf"), float("nan")
    gamma, keep = torch.ones(C), [1, 3, 5]
    for out in (dtype, "e4m3"):
        Y = torch.zeros(6, C, device=DEV).to(N.TORCH[out])
        scales = torch.zeros(6, device=DEV) if out == "e4m3" else None
        B.dsattn_rmsnorm(6, C, x.to(DEV), Y, gamma=gamma.to(DEV), scales=scales, io_dtype=N.CODE[dtype],
                         out_dtype=N.CODE[out], eps=0.0)
        torch.cuda.synchronize()
        y = Y.cpu().float()
        assert y[0].isnan().all() and y[4].isnan().all() and y[2, C // 2].isnan()
        if out == "e4m3":
            assert scales[[0, 2, 4]].isnan().all()
        else:
            assert (y[2].nan_to_num(0.0) == 0).all()
        N.check(3, C, dtype, out, x[keep], None, gamma, 0.0, None, Y[keep], None if scales is None else scales[keep])
