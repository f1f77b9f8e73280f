"""dsattn_linear_act of operands in 8 bits whose products cancel: the sums' bits, in every kernel.

The numbers are whole, and the sizes of a row's products add up to less than 2^24, so that a sum in fp32 is exact in any
order and its output is the formula's, rounded once.  Without DSATTN_FLAG_FP32_SUMS a bf16 output of the kernels on tiles of
64 rows or more may be off by what the header gives: 2^-13 of the largest product among 64 neighbouring channels, for
each of them (test_linear_act.py has the sum of that, `cut`)."""
import pytest
import torch

import test_linear_act as L
from paper_2406_16260_amd import binding as B
from test_linear_act_kernels import tile_of

DEV = "cuda:0"
FP32_SUMS = B.DSATTN_FLAG_FP32_SUMS
# (rows, c_in, c_out, rows of the tile without the flag, and with it)
SIZES = [(65, 320, 129, 32, 32), (700, 320, 1032, 64, 64), (20000, 256, 1000, 128, 128), (12000, 640, 1032, 256, 128)]


def outliers(M, K, N, sets, seed):
    """Small whole numbers, and pairs of channels whose products are as large as they come and cancel."""
    g = torch.Generator(device=DEV).manual_seed(seed)

    def whole(*s):
        return torch.randint(-3, 4, s, generator=g, device=DEV).float()

    x, w = whole(M, K), [whole(N, K) for _ in range(sets)]
    for i in range(8):
        at = K // 8 * i + i  # (pairs within a group of channels, and across groups)
        x[:, at], x[:, (at + 1 + 9 * i) % K] = 448.0, 448.0
        for k, a in enumerate(w):
            a[:, at], a[:, (at + 1 + 9 * i) % K] = 448.0, -448.0
    assert (x.abs() @ w[0].abs().t()).max().item() < 2 ** 24
    return {"X": x.to(torch.float8_e4m3fn), "W": [a.to(torch.float8_e4m3fn) for a in w], "sx": None, "sw": None, "b": None,
            "R": None}


def product(t, M, K, N, out, flags):
    Y = torch.full((M, N), float("nan"), device=DEV, dtype=L.TORCH[out])
    B.dsattn_linear_act(M, K, N, t["X"], t["W"], Y, io_dtype=B.DSATTN_E4M3, out_dtype=L.CODE[out], flags=flags)
    torch.cuda.synchronize()
    return Y


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,tile,wide", SIZES)
def test_fp32_sums_keep_what_cancelling_products_leave(M, K, N, tile, wide):
    print(f"[case] fp32 sums of {M} x {K} x {N}", flush=True)
    t = outliers(M, K, N, 1, M)
    exact = t["X"].double() @ t["W"][0].double().t()
    assert tile_of(M, K, N, "e4m3", "bf16", flags=FP32_SUMS) == wide
    assert torch.equal(product(t, M, K, N, "bf16", FP32_SUMS), exact.bfloat16())
    for flags in (0, FP32_SUMS):
        assert torch.equal(product(t, M, K, N, "f32", flags), exact.float())
    assert torch.equal(product(t, M, K, N, "bf16", FP32_SUMS | B.DSATTN_FLAG_FORCE_GENERIC), exact.bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,tile,wide", SIZES)
def test_gated_fp32_sums(M, K, N, tile, wide):
    t = outliers(M, K, N, 2, M + 1)
    z = [t["X"].double() @ w.double().t() for w in t["W"]]
    assert tile_of(M, K, N, "e4m3", "bf16", gated=True, flags=FP32_SUMS) == wide
    # (the product of two whole numbers below 2^24 is rounded in fp32, 2^-24, and to bf16)
    y, want = product(t, M, K, N, "bf16", FP32_SUMS).double(), z[0] * z[1]
    assert ((y - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -23)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,tile,wide", SIZES)
def test_without_the_flag_the_loss_is_within_its_bound(M, K, N, tile, wide):
    t = outliers(M, K, N, 1, M + 2)
    assert tile_of(M, K, N, "e4m3", "bf16") == tile
    y, exact = product(t, M, K, N, "bf16", 0).double(), t["X"].double() @ t["W"][0].double().t()
    if tile == 32:
        assert torch.equal(y, exact.bfloat16().double())
    bound = L.cut(t["X"].double(), t["W"][0].double())
    assert ((y - exact).abs() <= bound + (bound + exact.abs()) * 2.0 ** -8).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,gated", [(12000, 640, 1032, False), (12000, 640, 1032, True), (700, 320, 1032, True), (3, 128, 72, False),
                                         (20000, 256, 1000, False), (5, 40, 9, True)])
@pytest.mark.parametrize("act,bias,residual,scaled", [("none", True, True, True), ("gelu", False, False, True), ("silu", "first", True, False)])
def test_epilogues_with_fp32_sums(M, K, N, gated, act, bias, residual, scaled):
    """Against the formula within fp32's bounds, which the reference of an fp32 output has."""
    t = L.inputs(M, K, N, "e4m3", "bf16", M + N, gated, bias, residual, scaled)
    Y = torch.full((M, N), float("nan"), device=DEV, dtype=torch.bfloat16)
    L.call(t, M, K, N, "e4m3", "bf16", act, Y, FP32_SUMS)
    torch.cuda.synchronize()
    y, tol = L.reference(t, act, "f32")
    half = 2.0 ** -8
    assert ((Y.double() - y).abs() <= tol * (1 + half) + half * y.abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("e4m3", "f32")])
@pytest.mark.parametrize("M,K,N", [(65, 320, 129), (700, 320, 1032), (12000, 640, 1032)])
def test_the_flag_changes_nothing_else(M, K, N, dtype, out):
    t = L.inputs(M, K, N, dtype, out, 3, False, True, True, True)
    Y = [torch.empty(M, N, device=DEV, dtype=L.TORCH[out]) for _ in range(2)]
    for y, flags in zip(Y, (0, FP32_SUMS)):
        L.call(t, M, K, N, dtype, out, "silu", y, flags)
    torch.cuda.synchronize()
    assert torch.equal(Y[0], Y[1])


def test_the_kernels_with_and_without_the_flag():
    for M, K, N, tile, wide in SIZES:
        assert tile_of(M, K, N, "e4m3", "bf16") == tile and tile_of(M, K, N, "e4m3", "bf16", flags=FP32_SUMS) == wide
        for dtype, out in (("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("e4m3", "f32")):
            assert tile_of(M, K, N, dtype, out) == tile_of(M, K, N, dtype, out, flags=FP32_SUMS)
