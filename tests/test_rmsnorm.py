"""dsattn_rmsnorm: refusals on the host, and parity with the formula in 64 bits.

Tolerances: s = x + r is one fp32 rounding (2^-24), rounded once more where it is written.  The sum of
squares is of positive numbers: its relative error is at most its depth, C / 64 additions a lane and ten
joins, times 2^-24, and half of that after the root; the root, the reciprocal and the products add eight
roundings.  The output's own rounding is half a step: 2^-8 relative in bf16, 2^-4 in e4m3 and never less
than half of e4m3's smallest step, 2^-10."""
import ctypes

import pytest
import torch

from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
CODE = {"f32": B.DSATTN_F32, "bf16": B.DSATTN_BF16, "e4m3": B.DSATTN_E4M3}


def half_step(t):
    return torch.finfo(TORCH[t]).eps / 2


def inputs(rows, C, dtype, seed, residual):
    g = torch.Generator().manual_seed(seed)
    size = torch.exp(2.0 * torch.randn(rows, 1, generator=g))
    x = (torch.randn(rows, C, generator=g) * size).to(TORCH[dtype])
    r = torch.randn(rows, C, generator=g).to(TORCH[dtype]) if residual else None
    gamma = 1.0 + 0.3 * torch.randn(C, generator=g)
    return x, r, gamma


def formula(x, r, gamma, eps):
    s = x.double() if r is None else x.double() + r.double()
    y = s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    return s, y if gamma is None else y * gamma.double()


def check(rows, C, dtype, out, x, r, gamma, eps, S, Y, scales, mag=None):
    s, y = formula(x, r, gamma, eps)
    u = 2.0 ** -24 * (C / 128 + 13)
    if S is not None:
        tol = (s.abs() + 1e-300) * (half_step(dtype) + (2.0 ** -24 if dtype == "bf16" else 0.0)) * (1 + 1e-6)
        assert ((S.cpu().double() - s).abs() <= tol).all()
    got = Y.cpu().float().double()
    # an fp32 sum of operands that cancel is off by half a step of the operands' size at most
    lost = 2.0 ** -24 * (y / s).abs().nan_to_num(0.0) * ((x.double().abs() + r.double().abs()) if r is not None else 0.0)
    if out == "e4m3":
        want = y.abs().amax(-1) / 448
        sc = scales.cpu().double()
        assert ((sc - want).abs() <= want * 2 * u + 2.0 ** -126).all()
        z = y / sc[:, None]
        tol = torch.maximum(z.abs() * 2.0 ** -4, torch.full_like(z, 2.0 ** -10)) * (1 + 1e-6) + z.abs() * u + lost / sc[:, None]
        assert ((got - z).abs() <= tol).all()
    else:
        tol = y.abs() * (u + (half_step(out) if out == "bf16" else 0.0)) * (1 + 1e-6) + lost
        assert ((got - y).abs() <= tol).all()


def run(rows, C, dtype, out, seed, residual=True, affine=True, want_sum=True, eps=1e-6):
    x, r, gamma = inputs(rows, C, dtype, seed, residual)
    gamma = gamma if affine else None
    dx, dr, dg = (None if t is None else t.to(DEV) for t in (x, r, gamma))
    S = torch.full_like(dx, float("nan")) if want_sum else None
    Y = torch.full((rows, C), float("nan"), device=DEV).to(TORCH[out])
    scales = torch.full((rows,), float("nan"), device=DEV) if out == "e4m3" else None
    print(f"[case] rmsnorm {rows} x {C} {dtype} -> {out}, residual {residual}, gamma {affine}, sum {want_sum}", flush=True)
    B.dsattn_rmsnorm(rows, C, dx, Y, residual=dr, gamma=dg, sum_out=S, scales=scales, io_dtype=CODE[dtype],
                     out_dtype=CODE[out], eps=eps)
    torch.cuda.synchronize()
    check(rows, C, dtype, out, x, r, gamma, eps, S, Y, scales)
    return dx, dr, dg, S, Y, scales


ROWS_C = [(1, 1), (3, 7), (5, 8), (2, 31), (17, 40), (1000, 64), (33, 80), (129, 96), (66, 128), (7, 160), (5, 250),
          (9, 320), (3, 636), (70, 12), (33, 36), (5, 130), (4, 530), (3, 1030), (3, 1866), (2, 3996), (2, 4098), (2, 10004), (1, 16396), (31, 640), (40, 1280), (2, 1284), (11, 2560), (6, 4096), (4, 5120), (3, 8192), (2, 9999),
          (3, 16384), (2, 20000), (1, 65536)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("rows,C", ROWS_C)
def test_against_the_formula(rows, C, dtype, out):
    run(rows, C, dtype, out, 100 + rows + C)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [8, 64, 320, 1280, 9999])
@pytest.mark.parametrize("residual,affine,want_sum", [(False, False, False), (False, True, True), (True, False, False)])
@pytest.mark.parametrize("dtype,out", [("f32", "e4m3"), ("bf16", "bf16")])
def test_optional_tensors(C, residual, affine, want_sum, dtype, out):
    run(19, C, dtype, out, 7, residual, affine, want_sum)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [40, 1280, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(C, dtype):
    rows = 37
    x, r, gamma = inputs(rows, C, dtype, 11, True)
    dx, dr, dg = x.to(DEV), r.to(DEV), gamma.to(DEV)
    # the sum over the residual, the output over the input
    B.dsattn_rmsnorm(rows, C, dx, dx, residual=dr, gamma=dg, sum_out=dr, io_dtype=CODE[dtype])
    torch.cuda.synchronize()
    check(rows, C, dtype, dtype, x, r, gamma, 1e-6, dr, dx, None)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [24, 64, 320, 1280, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_zeros_infinities_and_nan(C, dtype):
    rows = 6
    x, _, gamma = inputs(rows, C, dtype, 5, False)
    x[0] = 0
    x[2, C // 2] = float("inf")
    x[4, C - 1] = float("nan")
    for out in (dtype, "e4m3"):
        Y = torch.zeros(rows, C, device=DEV).to(TORCH[out])
        scales = torch.zeros(rows, device=DEV) if out == "e4m3" else None
        B.dsattn_rmsnorm(rows, C, x.to(DEV), Y, gamma=gamma.to(DEV), scales=scales, io_dtype=CODE[dtype],
                         out_dtype=CODE[out])
        torch.cuda.synchronize()
        y = Y.cpu().float()
        assert (y[0] == 0).all()
        assert y[4].isnan().all() and y[2, C // 2].isnan()
        if out == "e4m3":
            assert scales[0].item() == 2.0 ** -126 and scales[2].isnan() and scales[4].isnan()
            assert y[2].isnan().all()
        else:
            assert (y[2].nan_to_num(0.0) == 0).all()
        keep = [1, 3, 5]
        check(3, C, dtype, out, x[keep], None, gamma, 1e-6, None, Y[keep], None if scales is None else scales[keep])


@pytest.mark.gpu
def test_rows_do_not_depend_on_their_number():
    """A row's result is the same alone and among others, and rows around it are left alone."""
    for C, dtype, out in ((320, "bf16", "bf16"), (1280, "bf16", "e4m3"), (640, "f32", "f32")):
        dx, dr, dg, S, Y, scales = run(700, C, dtype, out, 3)
        y1 = torch.zeros(1, C, device=DEV).to(TORCH[out])
        s1 = torch.zeros(1, device=DEV) if out == "e4m3" else None
        B.dsattn_rmsnorm(1, C, dx[321:322].contiguous(), y1, residual=dr[321:322].contiguous(), gamma=dg, scales=s1,
                         io_dtype=CODE[dtype], out_dtype=CODE[out])
        torch.cuda.synchronize()
        tol = 2.0 ** -22 if out == "f32" else 0.13 if out == "e4m3" else 2.0 ** -7
        assert ((y1.float() - Y[321:322].float()).abs() <= tol * Y[321:322].float().abs() + 1e-30).all()


def _desc(**kw):
    d = dict(rows=4, channels=64, io_dtype=B.DSATTN_BF16, out_dtype=B.DSATTN_BF16, eps=1e-6)
    d.update(kw)
    return B.DsattnRmsDesc(**d)


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(rows=-1), dict(rows=1 << 31), dict(channels=0), dict(channels=(1 << 20) + 1), dict(io_dtype=2),
    dict(io_dtype=3), dict(out_dtype=0), dict(io_dtype=0), dict(out_dtype=5), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf"))])
def test_bad_descriptors_are_refused(kw):
    lib = B.load()
    assert lib.dsattn_rmsnorm(ctypes.byref(_desc(**kw)), 0x10000, None, None, None, 0x20000, None, None) == B.DSATTN_EINVAL
    assert B.dsattn_last_error()


def test_bad_pointers_are_refused():
    lib = B.load()
    d, e = ctypes.byref(_desc()), ctypes.byref(_desc(out_dtype=B.DSATTN_E4M3))
    call = lib.dsattn_rmsnorm
    n = 4 * 64 * 2
    bad = [(None, 0x10000, None, None, None, 0x20000, None), (d, None, None, None, None, 0x20000, None),
           (d, 0x10000, None, None, None, None, None), (d, 0x10008, None, None, None, 0x20000, None),
           (d, 0x10000, 0x30004, None, None, 0x20000, None), (d, 0x10000, None, 0x30004, None, 0x20000, None),
           (d, 0x10000, None, None, 0x30008, 0x20000, None), (d, 0x10000, None, None, None, 0x20002, None),
           (d, 0x10000, None, None, None, 0x20000, 0x40000),               # scales without 8 bits
           (e, 0x10000, None, None, None, 0x20000, None),                  # 8 bits without scales
           (e, 0x10000, None, None, None, 0x20000, 0x40002),               # misaligned scales
           (d, 0x10000, None, None, None, 0x10010, None),                  # Y half over X
           (d, 0x10000, 0x30000, None, 0x30000 + n - 16, 0x20000, None),   # sum half over the residual
           (d, 0x10000, None, None, 0x20000, 0x20000, None),               # sum and Y the same
           (e, 0x10000, None, None, None, 0x10000, 0x40000),               # in place with another type
           (d, 0x10000, None, 0x20000, None, 0x20000, None),               # Y over gamma
           (e, 0x10000, None, None, None, 0x20000, 0x10000)]               # scales over X
    for args in bad:
        assert call(*args, None) == B.DSATTN_EINVAL, args


def test_binding_checks_tensors():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for kw in (dict(X=torch.zeros(4, 63, dtype=torch.bfloat16)), dict(X=x.float()), dict(Y=x.float()),
               dict(gamma=torch.zeros(63)), dict(gamma=x[0]), dict(sum_out=x[:3]), dict(scales=torch.zeros(5)),
               dict(residual=x.t()), {}):  # (the last: on the host)
        args = {"X": x, "Y": x, **kw}
        with pytest.raises(ValueError, match="dsattn_rmsnorm"):
            B.dsattn_rmsnorm(4, 64, **args)
