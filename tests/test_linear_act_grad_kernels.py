"""dsattn_linear_act_backward at sizes that each reach kernels of their own, against the formula: dz of many rows with every
activation (tiles of 256 x 128), weights' gradients in tiles of 256 x 256 whose rows are split, with and without a column
of tiles that is half empty, fp32 in tiles of 128 x 128; and what lies behind a workspace."""
import pytest
import torch

import test_linear_act_grad as G
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [(a, g) for a in G.ACTS for g in (False, True) if g or a != "none"])
@pytest.mark.parametrize("M,K,N", [(8200, 1032, 1288), (4100, 640, 2568), (512, 2048, 11008)])
def test_dz_of_many_rows(M, K, N, act, gated):
    G.run(M, K, N, "bf16", act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,act,gated", [
    (8200, 1032, 1288, "silu", True),      # 4 splits, the last column of tiles 8 wide
    (10000, 512, 2048, "gelu", True),      # 8 splits, the last of them shorter, whole tiles
    (40960, 640, 2560, "gelu", True),      # 4 splits, half a tile left
    (25920, 5120, 1280, "none", False),    # 5 splits
    (4096, 1280, 5120, "none", False),     # 2 splits
    (12345, 1400, 2568, "none", False),
    (30001, 640, 1288, "none", True)])
def test_weights_of_many_rows(M, K, N, act, gated):
    G.run(M, K, N, "bf16", act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("gelu", False), ("silu", True), ("gelu_tanh", True), ("relu", False), ("none", True)])
@pytest.mark.parametrize("M,K,N", [(6000, 640, 1280), (4097, 1288, 2564), (9001, 328, 644), (8192, 1024, 1024)])
def test_fp32_in_large_tiles(M, K, N, act, gated):
    G.run(M, K, N, "f32", act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,gated", [("none", False), ("gelu", True), ("silu", False)])
@pytest.mark.parametrize("M,K,N,flags", [(1, 64, 320, 0), (33, 72, 4040, 0), (130, 320, 264, 0), (300, 1280, 640, 0), (350, 2056, 1096, 0),
                                         (1100, 1032, 1048, 0), (2050, 320, 328, 0), (4100, 640, 1288, 0), (8200, 1032, 1288, 0),
                                         (33, 31, 9, 0), (130, 96, 72, B.DSATTN_FLAG_FORCE_GENERIC)])
def test_nothing_behind_the_workspace_is_written(M, K, N, flags, act, gated, dtype):
    t = G.inputs(M, K, N, dtype, act, 3, gated, True)
    need = B.dsattn_linear_act_backward_workspace(M, K, N, n_w=len(t["W"]), act=G.ACTS[act], io_dtype=G.CODE[dtype], flags=flags)
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    outs = []
    for ws in (room[:need] if need else None, "own"):
        out = torch.empty_like(t["X"]), [torch.empty_like(w) for w in t["W"]], [torch.empty(N, device=DEV) for _ in t["W"]]
        print(f"[case] {M} x {K} x {N} {dtype} {act} gated {gated} flags {flags}", flush=True)
        G.call(t, M, K, N, dtype, act, *out, flags=flags, ws=ws)
        torch.cuda.synchronize()
        outs.append([out[0], *out[1], *out[2]])
    assert (room[need:] == 0xA5).all()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# Sizes by kernel: few rows; dX's contraction split; tiles of 64 and 128, one stage ahead and two, down the columns and along the
# rows; tiles of 256; weights' gradients in 1 to 20 splits; rows that are not whole 16-byte pieces.
EXACT = [(1, 8, 8), (1, 392, 5040), (2, 320, 8), (17, 40, 24), (33, 72, 4040), (63, 72, 136), (65, 128, 200), (100, 136, 3208), (130, 4104, 2056),
         (160, 1280, 1280), (160, 264, 2568), (257, 520, 72), (350, 2056, 1096), (500, 1288, 1304), (640, 640, 640), (700, 2560, 2568),
         (1000, 96, 320), (1100, 1032, 1048), (2050, 320, 328), (2500, 1288, 1272), (4096, 1280, 5120), (4100, 640, 1288), (5000, 1280, 2560),
         (8200, 1032, 1288), (9001, 328, 640), (10000, 512, 2048), (12345, 1400, 2568), (25920, 1280, 648), (30001, 640, 1288),
         (40960, 320, 320), (3, 5, 7), (33, 31, 9), (129, 65, 130), (2000, 31, 9)]


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("none", False), ("none", True), ("relu", False), ("relu", True)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", EXACT)
def test_whole_numbers_come_out_exact(M, K, N, dtype, act, gated):
    """Inputs of -1, 0 and 1: z, dz (up to 256, what bf16 holds) and every sum (below 2^24) are whole numbers without rounding, so that
    nothing but the outputs' own rounding is allowed, and a row or a stage that is left out or taken twice is seen in
    any size.  A relu at 0 has a slope of 0 on both sides."""
    g = torch.Generator(device=DEV).manual_seed(M + K + N)
    sets, dt = 2 if gated else 1, G.TORCH[dtype]

    def whole(*shape):
        return torch.randint(-3, 4, shape, generator=g, device=DEV).div(2, rounding_mode="trunc").clamp(-1, 1)

    x, dy, w, b = whole(M, K), whole(M, N), [whole(N, K) for _ in range(sets)], [whole(N) for _ in range(sets)]
    if K > 600:  # (a quarter of the numbers only, so that sums of 5,120 stay below 256)
        w = [v * (torch.randint(0, 4, v.shape, generator=g, device=DEV) == 0) for v in w]
    t = {"X": x.to(dt), "dY": dy.to(dt), "W": [v.to(dt) for v in w], "b": [v.float() for v in b]}
    xd, z = x.double(), [x.double() @ v.double().t() + c.double() for v, c in zip(w, b)]
    on = (z[0] > 0).double() if act == "relu" else torch.ones_like(z[0])
    dz = [dy * z[1] * on, dy * z[0] * on] if gated else [dy * on]
    assert all(v.abs().max() <= 256 for v in dz)
    want = [sum(v @ u.double() for v, u in zip(dz, w)), *[v.t() @ xd for v in dz], *[v.sum(0) for v in dz]]
    assert all(v.abs().max() < 1 << 24 for v in want)
    out = [torch.full((M, K), float("nan"), device=DEV).to(dt), *[torch.full((N, K), float("nan"), device=DEV).to(dt) for _ in w],
           *[torch.full((N,), float("nan"), device=DEV) for _ in w]]
    print(f"[case] {M} x {K} x {N} {dtype} {act} gated {gated}", flush=True)
    G.call(t, M, K, N, dtype, act, out[0], out[1:1 + sets], out[1 + sets:])
    torch.cuda.synchronize()
    for k, (a, v) in enumerate(zip(out, want)):
        assert torch.equal(a, v.float().to(a.dtype)), k
