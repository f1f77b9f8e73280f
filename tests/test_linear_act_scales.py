"""dsattn_linear_act with scales whose product is none of fp32's numbers, in every kernel."""
import pytest
import torch

import test_linear_act as L
from paper_2406_16260_amd import binding as B
from test_linear_act_kernels import tile_of

DEV = "cuda:0"
# (rows, c_in, c_out, flags, rows of the tile): every kernel; ungated, bf16 operands and e4m3 ones
SIZES = [(5, 320, 1032, B.DSATTN_FLAG_FORCE_GENERIC, 0), (65, 320, 1032, 0, 32), (700, 320, 1032, 0, 64), (20000, 256, 1000, 0, 128),
         (12000, 640, 1032, 0, 256)]


def sized(dtype, out):
    for M, K, N, flags, tile in SIZES:
        got = tile_of(M, K, N, dtype, out, flags=flags)
        if (dtype, out) != ("e4m3", "f32"):
            assert got == tile
        yield M, K, N, flags


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_scales_are_applied_one_after_the_other(out, gated):
    """(acc x_scale) w_scale is one of fp32's and bf16's numbers, x_scale w_scale is not."""
    for M, K, N, flags in sized("e4m3", out):
        print(f"[case] scales of {M} x {K} x {N} -> {out}, gated {gated}, flags {flags}", flush=True)
        for a, sx, sw in ((2.0 ** 8, 2.0 ** -80, 2.0 ** -70), (2.0 ** -9, 2.0 ** 68, 2.0 ** 68), (0.0, 2.0 ** 70, 2.0 ** 70)):
            x, w = torch.full((M, K), a, device=DEV), torch.full((N, K), a, device=DEV)
            want = K * a * a * sx * sw
            # the value's product is one (or, of zeros, zero)
            v, sv = torch.zeros(N, K, device=DEV), torch.full((N,), 1.0 / (a * sx) if a else 1.0, device=DEV)
            v[:, K - 1] = 1.0
            e = torch.float8_e4m3fn
            Ws = [w.to(e), v.to(e)] if gated else [w.to(e)]
            sws = [torch.full((N,), sw, device=DEV), sv] if gated else [torch.full((N,), sw, device=DEV)]
            Y = torch.full((M, N), float("nan"), device=DEV, dtype=L.TORCH[out])
            B.dsattn_linear_act(M, K, N, x.to(e), Ws, Y, x_scales=torch.full((M,), sx, device=DEV), w_scales=sws,
                                io_dtype=B.DSATTN_E4M3, out_dtype=L.CODE[out], flags=flags)
            torch.cuda.synchronize()
            assert (Y.double() == want).all(), (a, sx, sw, Y[0, 0].item(), want)
