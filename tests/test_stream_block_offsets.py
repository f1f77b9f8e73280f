"""The operators of a streaming block on tensors whose offsets pass 32 bits, in the types and forms that
test_stream_block_large.py leaves out, against the formulas in 64 bits."""
import pytest
import torch

import test_linear_act as L
import test_rmsnorm as N
import test_sink_attn as S
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"


def filled(*shape, dtype, seed, size=1.0):
    """Normal numbers, without a tensor of four times the size in between."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.empty(*shape, dtype=dtype, device=DEV)
    flat = t.view(-1)
    step = 1 << 27
    for at in range(0, flat.numel(), step):
        n = min(step, flat.numel() - at)
        flat[at:at + n] = (size * torch.randn(n, generator=g, device=DEV)).to(dtype)
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out,gated,c_in,c_out,rows", [
    ("f32", "f32", False, 320, 2048, 600_000), ("f32", "f32", True, 2048, 320, 600_000),
    ("e4m3", "bf16", True, 4096, 512, 1_100_000), ("e4m3", "bf16", True, 256, 4096, 600_000),
    ("e4m3", "f32", False, 4096, 320, 1_100_000), ("e4m3", "f32", True, 256, 2048, 600_000),
    ("bf16", "bf16", True, 4096, 512, 600_000), ("bf16", "f32", True, 256, 2048, 600_000)])
def test_linear_act_of_more_than_4_gib(dtype, out, gated, c_in, c_out, rows):
    print(f"[case] linear_act {rows} x {c_in} x {c_out} {dtype} -> {out}, gated {gated}", flush=True)
    eight = dtype == "e4m3"
    x = filled(rows, c_in, dtype=L.TORCH[dtype], seed=2, size=16.0 if eight else 1.0)
    w = [filled(c_out, c_in, dtype=L.TORCH[dtype], seed=3 + k, size=(100.0 if eight else 1.0) * c_in ** -0.5)
         for k in range(2 if gated else 1)]
    sx = torch.rand(rows, device=DEV) / 16 if eight else None
    sw = [torch.rand(c_out, device=DEV) / 100 for _ in w] if eight else None
    r = filled(rows, c_out, dtype=L.TORCH[out], seed=7)
    y = torch.empty(rows, c_out, dtype=L.TORCH[out], device=DEV)
    B.dsattn_linear_act(rows, c_in, c_out, x, w, y, residual=r, x_scales=sx, w_scales=sw, act=B.DSATTN_ACT_SILU,
                        io_dtype=L.CODE[dtype], out_dtype=L.CODE[out])
    torch.cuda.synchronize()
    at32 = [(1 << b) // (c * es) for b in (31, 32) for c, es in ((c_in, x.element_size()), (c_out, y.element_size()))]
    for at in [0, rows - 300] + [a - 150 for a in at32 if a + 150 <= rows]:
        t = {"X": x[at:at + 300], "W": w, "sx": None if sx is None else sx[at:at + 300], "sw": sw, "b": None,
             "R": r[at:at + 300]}
        want, tol = L.reference(t, "silu", out)
        assert ((y[at:at + 300].double() - want).abs() <= tol).all(), at


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "e4m3")])
@pytest.mark.parametrize("C", [1280, 9999])
def test_rmsnorm_of_more_than_4_gib(C, dtype, out):
    rows = (9 << 29) // C
    print(f"[case] rmsnorm {rows} x {C} {dtype} -> {out}", flush=True)
    x = filled(rows, C, dtype=N.TORCH[dtype], seed=1)
    y, s = torch.empty(rows, C, dtype=N.TORCH[out], device=DEV), torch.empty_like(x)
    scales = torch.empty(rows, device=DEV) if out == "e4m3" else None
    gamma = torch.ones(C, device=DEV)
    B.dsattn_rmsnorm(rows, C, x, y, residual=x, gamma=gamma, sum_out=s, scales=scales, io_dtype=N.CODE[dtype],
                     out_dtype=N.CODE[out])
    torch.cuda.synchronize()
    for at in (0, (1 << 30) // C - 20, (1 << 31) // C - 20, rows - 40):
        part = x[at:at + 40].cpu()
        N.check(40, C, dtype, out, part, part, gamma.cpu(), 1e-6, s[at:at + 40], y[at:at + 40],
                None if scales is None else scales[at:at + 40])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T,h,window", [("bf16", 1, 8, 1100), ("bf16", 3, 16, 1100), ("bf16", 80, 8, 60), ("bf16", 80, 8, 1100),
                                              ("f32", 1, 8, 600), ("f32", 20, 8, 600), ("f32", 70, 8, 60)])
def test_sink_caches_of_more_than_4_gib(dtype, T, h, window):
    """Some positions of a large problem against the definition."""
    P, hk, D, sinks = 3000, 8, 80, 4
    ring = 1200 if dtype == "bf16" else 650
    print(f"[case] sink {T} x {P}, {h} on {hk} x {D}, window {window}, ring {ring} {dtype}", flush=True)
    t = S.TORCH[dtype]
    Kc, Vc = (filled(1, sinks + ring, P, hk * D, dtype=t, seed=s) for s in (5, 6))
    q = filled(1, T, P, h * D, dtype=t, seed=7)
    k, v = (filled(1, T, P, hk * D, dtype=t, seed=s) for s in (8, 9))
    few = torch.tensor([0, 1, 1499, 2300, 2999], device=DEV)
    c = S.case(dtype, T=T, P=len(few), h=h, hk=hk, D=D, sinks=sinks, window=window, ring=ring)
    s = S.Stream(c, 0)
    s.start = [5000]
    s.Q, s.K, s.V, s.Kc, s.Vc = (x.index_select(2, few).cpu() for x in (q, k, v, Kc, Vc))
    start = torch.full((1,), 5000, dtype=torch.int32, device=DEV)
    O = torch.zeros_like(q)
    shape = (1, T, P, h, hk, D, sinks, window, ring)
    space = torch.empty(B.dsattn_sink_workspace(*shape, io_dtype=S.CODE[dtype]), dtype=torch.uint8, device=DEV)
    B.dsattn_sink_forward(*shape, q, k, v, O, Kcache=Kc, Vcache=Vc, start=start, workspace=space, io_dtype=S.CODE[dtype])
    torch.cuda.synchronize()
    ref, tol = s.reference(D ** -0.5)
    assert ((O.index_select(2, few).cpu().double() - ref).abs() <= tol).all()
    Kw, Vw = s.caches()
    assert S.same_bits(Kc.index_select(2, few), Kw) and S.same_bits(Vc.index_select(2, few), Vw)
