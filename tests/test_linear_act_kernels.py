"""dsattn_linear_act by the kernel that a size takes: which one it is, and parity with the formula in 64 bits where
the persistent kernel is gated, has every activation, or lacks what is optional.

Tolerances are those of test_linear_act.py."""
import ctypes

import pytest
import torch

import test_linear_act as L
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"


def tile_of(M, K, N, dtype, out, gated=False, flags=0):
    """Rows of the tile that the library takes for a size, which names the kernel; 0: the vector kernel."""
    return B.dsattn_linear_act_info(M, K, N, n_w=2 if gated else 1, io_dtype=L.CODE[dtype], out_dtype=L.CODE[out],
                                    flags=flags)["tile_m"]


STREAMED = [("bf16", "bf16"), ("bf16", "f32"), ("e4m3", "bf16")]
# gated; some with several tiles a workgroup, rows and channels that no tile divides, channels that are no 16-byte pieces
GATED = [(12000, 640, 1032), (8200, 1280, 520), (20000, 2048, 515), (8100, 2560, 1023), (28013, 768, 1037)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", STREAMED)
@pytest.mark.parametrize("M,K,N", GATED)
def test_gated_products_on_persistent_workgroups(M, K, N, dtype, out):
    assert tile_of(M, K, N, dtype, out, gated=True) == 256
    L.run(M, K, N, dtype, out, act="gelu", gated=True, residual=M % 2 == 1)
    L.run(M, K, N, dtype, out, act="silu", gated=True, residual=M % 2 == 0, bias=False, scaled=False)


@pytest.mark.gpu
@pytest.mark.parametrize("act", sorted(L.ACTS))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype,out", STREAMED)
@pytest.mark.parametrize("bias,residual,scaled", [(False, False, True), (True, True, False), ("first", True, True),
                                                  (True, False, True)])
def test_epilogues_on_persistent_workgroups(bias, residual, scaled, dtype, out, gated, act):
    M, K, N = 12003, 640, 1036
    assert tile_of(M, K, N, dtype, out, gated) == 256
    L.run(M, K, N, dtype, out, act, gated, bias, residual, scaled)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", STREAMED)
def test_a_gated_residual_in_place_on_persistent_workgroups(dtype, out):
    M, K, N = 12000, 640, 1032
    assert tile_of(M, K, N, dtype, out, gated=True) == 256
    t = L.inputs(M, K, N, dtype, out, 9, True, True, True, True)
    y, tol = L.reference(t, "gelu", out)
    Y = t["R"].clone()
    L.call(t, M, K, N, dtype, out, "gelu", Y, residual=Y)
    torch.cuda.synchronize()
    assert ((Y.double() - y).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", STREAMED)
def test_infinities_and_nan_of_gated_products_stay_in_their_rows(dtype, out):
    M, K, N = 12000, 640, 1032
    assert tile_of(M, K, N, dtype, out, gated=True) == 256
    t = L.inputs(M, K, N, dtype, out, 4, True, True, False, True)
    t["X"][1, 5] = t["X"][M - 1, K - 1] = float("nan")
    Y = torch.empty(M, N, device=DEV, dtype=L.TORCH[out])
    L.call(t, M, K, N, dtype, out, "silu", Y)
    torch.cuda.synchronize()
    y, tol = L.reference(t, "silu", out)
    bad = ~Y.double().isfinite()
    assert bad[1].all() and bad[M - 1].all() and bad.sum().item() == 2 * N
    assert ((Y.double() - y).abs() <= tol)[~bad].all()


# ---- the choice, on the host

# (rows, c_in, c_out, gated) -> rows of the tile, 0 for the vector kernel; bf16 output
PICKS = [(1, 320, 1280, False, 32), (160, 1280, 1280, False, 32), (700, 320, 1032, False, 64), (20000, 256, 1000, False, 128),
         (12000, 640, 1032, False, 256), (65, 320, 129, True, 32), (700, 320, 1032, True, 64), (3000, 256, 1000, True, 128),
         (12000, 640, 1032, True, 256), (5, 7, 3, False, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("M,K,N,gated,tile", PICKS)
def test_the_kernel_of_a_size(M, K, N, gated, tile, dtype):
    got = B.dsattn_linear_act_info(M, K, N, n_w=2 if gated else 1, io_dtype=L.CODE[dtype])
    assert got["tile_m"] == tile and got["kernel"] == (1 if tile else 0)
    es, n = 1 if dtype == "e4m3" else 2, N * (2 if gated else 1)
    assert got["useful_flops"] == 2 * M * K * n
    assert got["algorithmic_bytes"] == (M + n) * K * es + 2 * M * N
    if tile:
        assert got["n_blocks"] == -(-M // tile) * -(-n // got["tile_n"]) and got["tile_k"] * es == 128
        assert got["block_threads"] in (128, 256, 512) and 0 < got["lds_bytes"] <= 160 << 10
    else:
        assert got["n_blocks"] == -(-M * N // 256) and got["block_threads"] == 256
    assert tile_of(M, K, N, dtype, "bf16", gated, B.DSATTN_FLAG_FORCE_GENERIC) == 0
    # no persistent kernel: fp32 tensors, and an fp32 output of 8-bit operands
    assert tile_of(M, K, N, "f32", "f32", gated) < 256 and tile_of(M, K, N, "e4m3", "f32", gated) < 256


def test_info_refuses_what_the_call_refuses():
    lib, info = B.load(), B.DsattnConvInfo()
    good = L._desc()
    assert lib.dsattn_linear_act_info(ctypes.byref(good), ctypes.byref(info)) == B.DSATTN_OK
    assert lib.dsattn_linear_act_info(ctypes.byref(good), None) == B.DSATTN_EINVAL
    assert lib.dsattn_linear_act_info(None, ctypes.byref(info)) == B.DSATTN_EINVAL
    for kw in (dict(rows=0), dict(c_in=0), dict(c_out=-1), dict(n_w=3), dict(act=9), dict(io_dtype=7), dict(out_dtype=2),
               dict(flags=2)):
        assert lib.dsattn_linear_act_info(ctypes.byref(L._desc(**kw)), ctypes.byref(info)) == B.DSATTN_EINVAL, kw
    with pytest.raises(B.DsattnError):
        B.dsattn_linear_act_info(0, 64, 32)


@pytest.mark.parametrize("kw", [dict(rows=(1 << 31) - 1, c_in=(1 << 31) - 1), dict(rows=(1 << 31) - 1, c_out=1 << 16),
                                dict(c_in=1 << 30, c_out=1 << 17), dict(rows=1 << 24, c_in=(1 << 31) - 1, c_out=1)])
def test_sizes_whose_bytes_pass_64_bits_are_refused(kw):
    lib, info = B.load(), B.DsattnConvInfo()
    d = L._desc(**{"io_dtype": B.DSATTN_F32, "out_dtype": B.DSATTN_F32, **kw})
    assert lib.dsattn_linear_act_info(ctypes.byref(d), ctypes.byref(info)) == B.DSATTN_EINVAL
    assert lib.dsattn_linear_act(ctypes.byref(d), 0x10000, None, L._vps(0x20000), None, None, None, 0x40000, None) == B.DSATTN_EINVAL
    big = L._desc(rows=(1 << 31) - 1, c_in=1 << 14, c_out=1 << 14, n_w=2)
    assert lib.dsattn_linear_act_info(ctypes.byref(big), ctypes.byref(info)) == B.DSATTN_OK and info.useful_flops > 0
