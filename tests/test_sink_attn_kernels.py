"""dsattn_sink_forward by the kernel that a shape takes: tiles shared by a workgroup at every head size, what a query
does not see in every kernel, and the choice itself.

Tolerances are those of test_sink_attn.py."""
import ctypes

import pytest
import torch

import test_sink_attn as S
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
VECTOR, STREAM, OWN_TILES, SHARED_TILES = 0, 1, 2, 3


def info(c, flags=0):
    return B.dsattn_sink_forward_info(c["B"], c["T"], c["P"], c["h"], c["hk"], c["D"], c["sinks"], c["window"], c["ring"],
                                      io_dtype=S.CODE[c["dtype"]], flags=flags)


TILE_DIMS = [D for D in S.DIMS if D % 8 == 0 and D <= 256]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", TILE_DIMS)
@pytest.mark.parametrize("window,tile", [(40, 32), (100, 32), (200, 64)])
def test_shared_tiles_of_every_head_dim(window, tile, D, dtype):
    """Rings that the attention fills on the way (roomy, or a stream's beginning) and that a kernel fills after it."""
    for start, ring in ((0, window), (0, window + 69), (13, window), (13, window + 69), (290, window), (290, window + 80)):
        c = S.case(dtype, T=70, P=2, h=2, D=D, sinks=3, window=window, ring=ring, start=start)
        got = info(c)
        assert got["kernel"] == SHARED_TILES and got["tile_frames"] == (32 if dtype == "f32" else tile)
        S.run(c, D + start)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 80, 136, 160, 256])
@pytest.mark.parametrize("h,hk,T", [(6, 2, 50), (3, 1, 130), (8, 8, 300), (20, 4, 33)])
def test_shared_tiles_of_shared_heads_and_ragged_streams(h, hk, T, D, dtype):
    for window in (33, 150):
        c = S.case(dtype, B=4, T=T, P=2, h=h, hk=hk, D=D, sinks=4, window=window, ring=window + T // 2,
                   start=[0, 7, 200, 60], counts=[T, T - 1, 1, 0])
        assert info(c)["kernel"] == SHARED_TILES
        S.run(c, T + D)


# kernel, whether it has parts, and a shape that takes it
HIDING = [(OWN_TILES, False, dict(T=40, P=2, h=2, D=64, window=20)),
          (OWN_TILES, False, dict(T=17, P=2, h=4, hk=2, D=200, window=25)),
          (SHARED_TILES, False, dict(T=70, P=2, h=2, D=80, window=60)),
          (SHARED_TILES, False, dict(T=70, P=2, h=2, D=160, window=90)),
          (SHARED_TILES, False, dict(T=90, P=2, h=4, hk=2, D=128, window=140)),
          (SHARED_TILES, True, dict(T=100, P=2, h=4, hk=2, D=64, window=3300)),
          (OWN_TILES, True, dict(T=7, P=2, h=8, hk=1, D=64, window=3000)),
          (STREAM, True, dict(T=3, P=2, h=1, D=128, window=5000)),
          (STREAM, False, dict(T=2, P=2, h=2, hk=1, D=40, window=30))]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kernel,parts,shape", HIDING)
def test_what_a_query_does_not_see_does_not_reach_it(kernel, parts, shape, dtype):
    """Infinities and NaN in a new frame (position 0) and in a cached one that the first queries see only (position 1):
    those that see them are no numbers, all others as without them."""
    T, P, w = shape["T"], shape["P"], shape["window"]
    start, hit = w + 100, T // 2
    last = min(10, T - 1)  # the first query that does not see the cached frame any more
    old = start - w + last
    for ring in (w, w + T):
        c = S.case(dtype, sinks=2, ring=ring, start=start, **shape)
        got = info(c)
        assert got["kernel"] == kernel and (got["splits"] > 1) == parts
        print(f"[case] sink {c}: infinities and NaN", flush=True)
        clean, tol = S.Stream(c, 1).reference(c["D"] ** -0.5)
        for tensor, value in (("V", "nan"), ("V", "inf"), ("K", "nan"), ("K", "inf")):
            s = S.Stream(c, 1)
            getattr(s, tensor)[0, hit, 0, :] = float(value)
            getattr(s, tensor + "c")[0, S.slot(old, 2, ring), 1, :] = float(value)
            O = torch.zeros(1, T, P, c["h"] * c["D"], dtype=S.TORCH[dtype], device=DEV)
            S.forward(s, c, O, s.Kc.to(DEV), s.Vc.to(DEV))
            torch.cuda.synchronize()
            bad = ~O.float().isfinite().cpu()
            want = torch.zeros(T, P, dtype=torch.bool)
            want[hit:, 0] = True
            want[:last, 1] = True
            if value == "nan" or tensor == "V":
                assert torch.equal(bad[0].all(-1), want) and torch.equal(bad[0].any(-1), want), (tensor, value)
            ok = ~want[None, :, :, None].expand_as(bad)
            assert ((O.cpu().double() - clean).abs() <= tol)[ok].all(), (tensor, value)


# ---- the choice, on the host

SHAPES = [(STREAM, False, dict(T=1, P=160, h=8, D=160, window=60)), (STREAM, True, dict(T=1, P=1, h=32, hk=8, D=128, window=4096)),
          (OWN_TILES, False, dict(T=7, P=160, h=8, D=80, window=60)), (OWN_TILES, True, dict(T=8, P=1, h=32, hk=8, D=128, window=4096)),
          (SHARED_TILES, False, dict(T=128, P=640, h=8, D=80, window=32)), (SHARED_TILES, True, dict(T=512, P=1, h=16, hk=4, D=128, window=4096)),
          (VECTOR, False, dict(T=40, P=3, h=2, D=100, window=60)), (VECTOR, False, dict(T=9, P=3, h=2, D=512, window=60))]


@pytest.mark.parametrize("kernel,parts,shape", SHAPES)
def test_the_kernel_of_a_shape(kernel, parts, shape):
    c = S.case("bf16", **shape)
    got = info(c)
    assert got["kernel"] == kernel and (got["splits"] > 1) == parts
    assert got["n_blocks"] >= 1 and got["block_threads"] in (256, 512) and 0 <= got["lds_bytes"] <= 160 << 10
    assert (got["tile_rows"] > 0) == (got["tile_frames"] > 0) == (kernel >= OWN_TILES)
    need = B.dsattn_sink_workspace(c["B"], c["T"], c["P"], c["h"], c["hk"], c["D"], c["sinks"], c["window"], c["ring"])
    assert need == (c["B"] * c["T"] * c["P"] * c["h"] * got["splits"] * (c["D"] + 4) * 4 if parts else 0)
    assert info(c, B.DSATTN_FLAG_FORCE_GENERIC)["kernel"] == VECTOR


def test_every_tested_shape_takes_the_kernel_that_it_is_for():
    for kernel, parts, shape in HIDING:
        for dtype in ("f32", "bf16"):
            got = info(S.case(dtype, sinks=2, **shape))
            assert got["kernel"] == kernel and (got["splits"] > 1) == parts, (dtype, shape, got)
    for D in TILE_DIMS:
        for window, tile in ((40, 32), (100, 32), (200, 64)):
            got = info(S.case("bf16", T=70, P=2, h=2, D=D, sinks=3, window=window))
            assert got["kernel"] == SHARED_TILES and got["tile_frames"] == tile


def test_info_refuses_what_the_call_refuses():
    lib, out = B.load(), B.DsattnSinkInfo()
    assert lib.dsattn_sink_forward_info(ctypes.byref(S._desc()), ctypes.byref(out)) == B.DSATTN_OK
    assert lib.dsattn_sink_forward_info(ctypes.byref(S._desc()), None) == B.DSATTN_EINVAL
    assert lib.dsattn_sink_forward_info(None, ctypes.byref(out)) == B.DSATTN_EINVAL
    for kw in S.BAD:
        assert lib.dsattn_sink_forward_info(ctypes.byref(S._desc(**kw)), ctypes.byref(out)) == B.DSATTN_EINVAL, kw
    with pytest.raises(B.DsattnError):
        B.dsattn_sink_forward_info(1, 1, 1, 3, 2, 64, 0, 4)


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_a_scale_beyond_fp32_in_powers_of_two_is_refused(scale):
    lib, out = B.load(), B.DsattnSinkInfo()
    assert lib.dsattn_sink_forward_info(ctypes.byref(S._desc(scale=scale)), ctypes.byref(out)) == B.DSATTN_EINVAL
    for good in (2.3e38, -3.4e38, 0.0):  # (the last two select 1 / sqrt(head_dim))
        assert lib.dsattn_sink_forward_info(ctypes.byref(S._desc(scale=good)), ctypes.byref(out)) == B.DSATTN_OK
