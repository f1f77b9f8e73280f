"""Rows of equal numbers of every size, and rows whose numbers differ in their last bits only, through dsattn_layernorm and its
backward pass.

A row of equal numbers has no spread: n is 0, y is beta rounded once, and 1 / sqrt(var + eps) is eps^-1/2.  Its formula is
that of a row of zeros, which is where the expected values come from (in 64 bits the mean of numbers of 1e36 is itself off by
1e20).  Differences of a row's numbers from its first one are exact in 64 bits, and the norm does not see such a shift."""
import pytest
import torch

import test_layernorm as N
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
SIZES = [1.0, 1000.1, 1.3e5, 7.7e9, 1.1e15, 9.3e19, 1.234e26, 1e26, 3.3e26, 1e30, 1e36, 2.9e38]
LENGTHS = [1, 3, 7, 63, 250, 320, 515, 1279, 1280, 4099, 9000, 16383, 20001]


def equal_rows(C, dtype, residual):
    """x, r: rows of either sign, and two ordinary ones between them."""
    s = torch.tensor([v * f for v in SIZES for f in (1.0, -1.0)])
    x = s[:, None].expand(-1, C).clone().to(N.TORCH[dtype])
    g = torch.Generator().manual_seed(C)
    ordinary = torch.randn(2, C, generator=g).to(N.TORCH[dtype])
    x = torch.cat([x[:5], ordinary[:1], x[5:], ordinary[1:]])
    r = None
    if residual:  # equal numbers too, half as large
        r = (0.5 * x.float()).to(N.TORCH[dtype])
        r[5], r[-1] = ordinary[1].flip(0), ordinary[0].flip(0)
        x[-3:-1], r[-3:-1] = x[:2], r[:2]  # (their sum would be infinite)
    return x, r, [i for i in range(len(x)) if i not in (5, len(x) - 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [1e-6, 1e-30])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("C", LENGTHS)
def test_rows_of_equal_numbers_are_beta(C, dtype, out, residual, eps):
    x, r, equal = equal_rows(C, dtype, residual)
    keep = [i for i in range(len(x)) if i not in equal]
    _, _, gamma, beta, _, _ = N.inputs(1, C, dtype, 9, False)
    rows = len(x)
    Y = torch.full((rows, C), float("nan"), device=DEV).to(N.TORCH[out])
    S = torch.empty(rows, C, device=DEV, dtype=N.TORCH[dtype])
    scales = torch.empty(rows, device=DEV) if out == "e4m3" else None
    B.dsattn_layernorm(rows, C, x.to(DEV), Y, residual=None if r is None else r.to(DEV), gamma=gamma.to(DEV), beta=beta.to(DEV),
                       sum_out=S, scales=scales, io_dtype=N.CODE[dtype], out_dtype=N.CODE[out], eps=eps)
    torch.cuda.synchronize()
    if out == "e4m3":
        zero = torch.zeros(len(equal), C, dtype=N.TORCH[dtype])
        N.check(dtype, out, zero, None, gamma, beta, eps, None, Y[equal], scales[equal])
    else:
        assert (Y[equal].cpu() == beta.to(N.TORCH[out])).all()
    some = None if scales is None else scales[keep]
    if C > 1:
        N.check(dtype, out, x[keep], None if r is None else r[keep], gamma, beta, eps, S[keep], Y[keep], some)


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", LENGTHS)
def test_gradients_of_rows_of_equal_numbers(C, dtype, residual):
    """Among them ordinary rows, whose dgamma they leave as it is."""
    x, r, equal = equal_rows(C, dtype, residual)
    rows = len(x)
    _, _, gamma, _, dy, ds = N.inputs(rows, C, dtype, 10, False)
    t = [v.to(DEV) for v in (x, gamma, dy, ds)]
    dX = torch.full((rows, C), float("nan"), device=DEV).to(N.TORCH[dtype])
    dg, db = (torch.full((C,), float("nan"), device=DEV) for _ in range(2))
    B.dsattn_layernorm_backward(rows, C, t[0], t[2], dX, residual=None if r is None else r.to(DEV), gamma=t[1], dsum=t[3], dgamma=dg,
                                dbeta=db, workspace=N.space(rows, C, dtype), io_dtype=N.CODE[dtype])
    torch.cuda.synchronize()
    x[equal] = 0
    if residual:
        r[equal] = 0
    want = N.gradients(x, r, gamma, 1e-6, dy, ds)
    N.near(dX.float(), want[0], N.half_step(dtype))
    N.near(dg, want[1])
    N.near(db, want[2])


@pytest.mark.gpu
@pytest.mark.parametrize("share", [0.001, 0.3, 0.5])
@pytest.mark.parametrize("size", [1.0, 1.3e5, 1.1e15, 1.234e26, 1e30, 1e36])
@pytest.mark.parametrize("C", [63, 320, 1280, 4099, 20001])
def test_rows_that_differ_in_a_last_bit(C, size, share):
    """Numbers that are one of two neighbours, with eps far below their variance.  What is left of the mean after the first time is
    half a unit of the last bit at most, so that the variance of whole units loses a bit or two of its sum's: twice the tolerance of
    rows whose mean is 0, and the differences from the row's first number as x."""
    g = torch.Generator().manual_seed(C)
    low = torch.full((4, C), size)
    pick = torch.rand(4, C, generator=g) < share
    pick[0], pick[1] = False, True
    pick[0, C // 2], pick[1, C // 3] = True, False
    pick[2, 0], pick[2, 1], pick[3, 0], pick[3, 1] = True, False, False, True
    x = torch.where(pick, torch.nextafter(low, torch.full_like(low, float("inf"))), low)
    _, _, gamma, beta, _, _ = N.inputs(1, C, "f32", 9, False)
    Y = torch.full((4, C), float("nan"), device=DEV)
    B.dsattn_layernorm(4, C, x.to(DEV), Y, gamma=gamma.to(DEV), beta=beta.to(DEV), io_dtype=B.DSATTN_F32, eps=0.0)
    torch.cuda.synchronize()
    d = x.double() - x[:, :1].double()
    unit = d.abs().max()
    d = d / unit
    _, _, n, _, tol, _ = N.normed(d, None, 0.0)
    y = n * gamma.double() + beta.double()
    tol = 2 * tol * gamma.double().abs() + 3 * N.U * ((n * gamma).abs() + beta.double().abs())
    off = (Y.cpu().double() - y).abs()
    assert (off <= tol).all(), f"{(off / tol).max().item()} of the tolerance"


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [65537, 999999, 1 << 20])
def test_the_longest_rows(C, dtype, residual):
    """Sums of 4,096 numbers a lane, whose first mean is off by some hundred units of the last bit."""
    test_rows_of_equal_numbers_are_beta(C, dtype, dtype, residual, 1e-6)
    test_gradients_of_rows_of_equal_numbers(C, dtype, residual)


@pytest.mark.gpu
@pytest.mark.parametrize("most", [1, 3, 1000, 1 << 20])
@pytest.mark.parametrize("C", [7, 63, 320, 1280, 4099, 20001])
def test_rows_of_the_smallest_numbers(C, most):
    """Whole multiples of 2^-149 have the norm of those whole numbers, eps 0 (twice the tolerance, as for rows that differ in a last bit:
    a mean of few units of the last bit is that far off before its rest is taken off)."""
    g = torch.Generator().manual_seed(C + most)
    x = torch.randint(0, most + 1, (5, C), generator=g).float()
    x[:, 0], x[:, 1] = 0.0, float(most)
    x[3:] = x[3:] - most // 2
    _, _, gamma, beta, _, _ = N.inputs(1, C, "f32", 9, False)
    Y = torch.full((5, C), float("nan"), device=DEV)
    tiny = torch.ldexp(x, torch.tensor(-149))
    assert torch.equal(tiny.double() * 2.0 ** 149, x.double())
    B.dsattn_layernorm(5, C, tiny.to(DEV), Y, gamma=gamma.to(DEV), beta=beta.to(DEV), io_dtype=B.DSATTN_F32, eps=0.0)
    torch.cuda.synchronize()
    _, _, n, _, tol, _ = N.normed(x, None, 0.0)
    y = n * gamma.double() + beta.double()
    tol = 2 * tol * gamma.double().abs() + 3 * N.U * ((n * gamma).abs() + beta.double().abs())
    off = (Y.cpu().double() - y).abs()
    assert (off <= tol).all(), f"{(off / tol).max().item()} of the tolerance"
