"""dsattn_layernorm and its backward pass: refusals on the host, the formulas against differences, and parity with them in 64 bits.

Tolerances, u = 2^-24.  s = x + r is off by one rounding, u (|x| + |r|) at most.  Its mean is taken off twice, so that what is
left of the mean's error is that of the sum of the differences d: n = C / 256 or 32 additions a lane, whichever is more, and
twelve joins, (n + 12) u mean|d|.  The variance has that depth too, half of it after the root; the root, the quotient and the
products add eight roundings.  An output's own rounding is half a step.  The backward pass's two means have the same depth
of their terms' sizes; sums over rows have rows / 1,024 additions a lane and 100 joins at most (64 rows a workgroup of long rows)."""
import ctypes

import pytest
import torch

from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
CODE = {"f32": B.DSATTN_F32, "bf16": B.DSATTN_BF16, "e4m3": B.DSATTN_E4M3}
U = 2.0 ** -24


def half_step(t):
    return torch.finfo(TORCH[t]).eps / 2 if t == "bf16" else 0.0


def inputs(rows, C, dtype, seed, residual, mean=0.5):
    g = torch.Generator().manual_seed(seed)
    size = torch.exp(2.0 * torch.randn(rows, 1, generator=g))
    x = ((torch.randn(rows, C, generator=g) + mean * torch.randn(rows, 1, generator=g)) * size).to(TORCH[dtype])
    r = torch.randn(rows, C, generator=g).to(TORCH[dtype]) if residual else None
    gamma, beta = 1.0 + 0.3 * torch.randn(C, generator=g), 0.5 * torch.randn(C, generator=g)
    dy, ds = (torch.randn(rows, C, generator=g).to(TORCH[dtype]) for _ in range(2))
    return x, r, gamma, beta, dy, ds


def depth(C):
    return max(32, C / 256) + 12


def normed(x, r, eps):
    """s, d, n, 1 / deviation, and the tolerances of n and (relative) of the last, in 64 bits."""
    s = x.double() if r is None else x.double() + r.double()
    es = torch.zeros_like(s) if r is None else U * (x.double().abs() + r.double().abs())
    C = x.shape[1]
    d = s - s.mean(-1, keepdim=True)
    var = (d * d).mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    n = d * rstd
    mean_d = d.abs().mean(-1, keepdim=True)
    # (the deviation follows an error of s at most as far as its mean size)
    rel = U * (depth(C) / 2 + 8) + (es * d.abs()).mean(-1, keepdim=True) / (var + eps)
    # (what the first mean is off by, depth u mean|s|, is rounded with d and in the mean of the differences)
    first = depth(C) * U * s.abs().mean(-1, keepdim=True)
    tol = (es + es.mean(-1, keepdim=True) + 4 * U * (d.abs() + first) + depth(C) * U * (mean_d + first)) * rstd + n.abs() * rel
    return s, d, n, rstd, tol, rel


def check(dtype, out, x, r, gamma, beta, eps, S, Y, scales=None):
    s, _, n, _, tol, _ = normed(x, r, eps)
    g = torch.ones(x.shape[1]).double() if gamma is None else gamma.double()
    b = torch.zeros(x.shape[1]).double() if beta is None else beta.double()
    y = n * g + b
    if S is not None:
        assert ((S.cpu().double() - s).abs() <= s.abs() * (half_step(dtype) + 2 * U)
                + (0 if r is None else U * (x.double().abs() + r.double().abs()))).all()
    got, tol = Y.cpu().float().double(), tol * g.abs() + 2 * U * ((n * g).abs() + b.abs())
    if out == "e4m3":
        sc = scales.cpu().double()
        want = y.abs().amax(-1) / 448
        assert ((sc - want).abs() <= tol.amax(-1) / 448 + 4 * U * want + 2.0 ** -126).all()
        z = y / sc[:, None]
        tol = tol / sc[:, None] + torch.maximum(z.abs() * 2.0 ** -4, torch.full_like(z, 2.0 ** -10)) * (1 + 1e-6) + 4 * U * z.abs()
        assert ((got - z).abs() <= tol).all()
        return
    off = (got - y).abs()
    tol = tol * (1 + half_step(out)) + half_step(out) * y.abs() + U * y.abs()
    assert (off <= tol).all(), f"{(off / tol).max().item()} of the tolerance"


def gradients(x, r, gamma, eps, dy, ds):
    """dx, dgamma, dbeta and their tolerances in fp32, in 64 bits."""
    _, _, n, rstd, en, rel = normed(x, r, eps)
    C, rows = x.shape[1], x.shape[0]
    g = torch.ones(C).double() if gamma is None else gamma.double()
    dy, ds = dy.double(), torch.zeros_like(n) if ds is None else ds.double()
    e = dy * g
    m0, m1 = e.mean(-1, keepdim=True), (e * n).mean(-1, keepdim=True)
    core = (e - m0 - n * m1) * rstd
    dn = depth(C)
    em0 = dn * U * e.abs().mean(-1, keepdim=True)
    em1 = dn * U * (e * n).abs().mean(-1, keepdim=True) + (e.abs() * en).mean(-1, keepdim=True)
    tol = rstd * (em0 + m1.abs() * en + n.abs() * em1 + 5 * U * (e.abs() + m0.abs() + (n * m1).abs())) + core.abs() * (rel + 4 * U)
    dx = core + ds
    long = (rows / 1024 + 100) * U
    return (dx, tol + U * (core.abs() + ds.abs())), ((dy * n).sum(0), (dy.abs() * en).sum(0) + long * (dy * n).abs().sum(0)), \
        (dy.sum(0), long * dy.abs().sum(0))


def near(got, want_tol, half=0.0):
    want, tol = want_tol
    off = (got.cpu().double() - want).abs()
    tol = tol * (1 + half) + half * want.abs()
    assert (off <= tol).all(), f"{(off / tol.clamp_min(1e-300)).max().item()} of the tolerance"


def run(rows, C, dtype, out, seed, residual=True, affine=True, want_sum=True, eps=1e-6, mean=0.5):
    x, r, gamma, beta, _, _ = inputs(rows, C, dtype, seed, residual, mean)
    gamma, beta = (gamma, beta) if affine else (None, None)
    dx, dr, dg, db = (None if t is None else t.to(DEV) for t in (x, r, gamma, beta))
    S = torch.full_like(dx, float("nan")) if want_sum else None
    Y = torch.full((rows, C), float("nan"), device=DEV).to(TORCH[out])
    scales = torch.full((rows,), float("nan"), device=DEV) if out == "e4m3" else None
    print(f"[case] layernorm {rows} x {C} {dtype} -> {out}, residual {residual}, affine {affine}, sum {want_sum}", flush=True)
    B.dsattn_layernorm(rows, C, dx, Y, residual=dr, gamma=dg, beta=db, sum_out=S, scales=scales, io_dtype=CODE[dtype],
                       out_dtype=CODE[out], eps=eps)
    torch.cuda.synchronize()
    check(dtype, out, x, r, gamma, beta, eps, S, Y, scales)


def space(rows, C, dtype):
    n = B.dsattn_layernorm_backward_workspace(rows, C, io_dtype=CODE[dtype])
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV)  # (NaN, wherever it is read before it is written)


def run_back(rows, C, dtype, seed, residual=True, affine=True, dsum=True, sums=True, eps=1e-6):
    x, r, gamma, beta, dy, ds = inputs(rows, C, dtype, seed, residual)
    gamma, ds = gamma if affine else None, ds if dsum else None
    d = {k: None if t is None else t.to(DEV) for k, t in (("x", x), ("r", r), ("g", gamma), ("dy", dy), ("ds", ds))}
    guard = torch.full((rows * C + 64,), 7.0, device=DEV).to(TORCH[dtype])
    dX = guard[:rows * C].view(rows, C)
    dg, db = (torch.full((C,), float("nan"), device=DEV) for _ in range(2)) if sums else (None, None)
    print(f"[case] layernorm_backward {rows} x {C} {dtype}, residual {residual}, gamma {affine}, dsum {dsum}, sums {sums}", flush=True)
    B.dsattn_layernorm_backward(rows, C, d["x"], d["dy"], dX, residual=d["r"], gamma=d["g"], dsum=d["ds"], dgamma=dg, dbeta=db,
                                workspace=space(rows, C, dtype) if sums else None, io_dtype=CODE[dtype], eps=eps)
    torch.cuda.synchronize()
    want = gradients(x, r, gamma, eps, dy, ds)
    near(dX.float(), want[0], half_step(dtype))
    assert (guard[rows * C:] == 7.0).all(), "written past the end"
    if sums:
        near(dg, want[1])
        near(db, want[2])
    return d, dX, dg, db


ROWS_C = [(1, 1), (3, 7), (5, 8), (2, 31), (17, 40), (1000, 64), (33, 80), (129, 96), (66, 128), (7, 160), (5, 250), (9, 320),
          (3, 636), (70, 12), (33, 36), (5, 130), (4, 530), (3, 1030), (3, 1866), (2, 3996), (2, 4098), (2, 10004), (1, 16396),
          (31, 640), (40, 1280), (2, 1284), (11, 2560), (6, 4096), (4, 5120), (3, 8192), (2, 9999), (3, 16384), (130, 20000),
          (1, 65536), (5000, 24), (9001, 72)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("rows,C", ROWS_C)
def test_against_the_formula(rows, C, dtype, out):
    run(rows, C, dtype, out, 100 + rows + C)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", ROWS_C)
def test_gradients_against_the_formula(rows, C, dtype):
    run_back(rows, C, dtype, 300 + rows + C)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [8, 64, 320, 1280, 9999, 20000])
@pytest.mark.parametrize("residual,affine,extra", [(False, False, False), (False, True, True), (True, False, False)])
@pytest.mark.parametrize("dtype,out", [("f32", "e4m3"), ("bf16", "bf16")])
def test_optional_tensors(C, residual, affine, extra, dtype, out):
    run(19, C, dtype, out, 7, residual, affine, extra)
    run_back(19, C, dtype, 8, residual, affine, extra, sums=extra)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [40, 1280, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(C, dtype):
    rows = 37
    x, r, gamma, beta, dy, ds = inputs(rows, C, dtype, 11, True)
    dx, dr, dg, db = x.to(DEV), r.to(DEV), gamma.to(DEV), beta.to(DEV)
    B.dsattn_layernorm(rows, C, dx, dx, residual=dr, gamma=dg, beta=db, sum_out=dr, io_dtype=CODE[dtype])
    torch.cuda.synchronize()
    check(dtype, dtype, x, r, gamma, beta, 1e-6, dr, dx)
    want = gradients(x, r, gamma, 1e-6, dy, ds)
    for which in range(4):
        t = [v.to(DEV) for v in (x, r, dy, ds)]
        sums = C <= (8192 if dtype == "f32" else 16384) or which == 3
        out = [torch.empty(C, device=DEV) for _ in range(2)] if sums else [None, None]
        B.dsattn_layernorm_backward(rows, C, t[0], t[2], t[which], residual=t[1], gamma=dg, dsum=t[3], dgamma=out[0], dbeta=out[1],
                                    workspace=space(rows, C, dtype), io_dtype=CODE[dtype])
        torch.cuda.synchronize()
        near(t[which].float(), want[0], half_step(dtype))
        if sums:
            near(out[0], want[1])
            near(out[1], want[2])


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 8, 9, 16, 17, 64, 129])
@pytest.mark.parametrize("C", [5, 60, 320, 1279, 2560, 8192, 9000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sums_of_few_rows(rows, C, dtype):
    """In one workgroup, or joined; to places aligned to four bytes; one of the two alone."""
    x, r, gamma, beta, dy, ds = inputs(rows, C, dtype, 400 + rows + C, True)
    want = gradients(x, r, gamma, 1e-6, dy, ds)
    t = [v.to(DEV) for v in (x, r, gamma, dy, ds)]
    wanted = [torch.full((C + 8,), 7.0, device=DEV) for _ in range(3)]
    dg, db, alone = (v[1 + i:1 + i + C] for i, v in enumerate(wanted))
    for dgamma, dbeta in ((dg, db), (None, alone)):
        dX = torch.empty_like(t[0])
        B.dsattn_layernorm_backward(rows, C, t[0], t[3], dX, residual=t[1], gamma=t[2], dsum=t[4], dgamma=dgamma, dbeta=dbeta,
                                    workspace=space(rows, C, dtype), io_dtype=CODE[dtype])
        torch.cuda.synchronize()
        near(dX.float(), want[0], half_step(dtype))
    near(dg, want[1])
    near(db, want[2])
    assert (alone == db).all()
    for i, v in enumerate(wanted):
        assert (v[:1 + i] == 7.0).all() and (v[1 + i + C:] == 7.0).all(), "written past the ends"


@pytest.mark.gpu
@pytest.mark.parametrize("C", [1, 7, 9, 65, 257, 515, 1279, 2049, 4099, 9999])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_at_odd_lengths(C, dtype):
    """The last 16 bytes of a row share numbers with those before."""
    test_in_place(C, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [1, 3, 6, 11, 63, 250, 320, 515, 636, 1284, 1863, 2049, 4097, 8191, 16383, 20001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_equal_numbers_have_no_spread(C, dtype):
    """A row of C times one number s of 8 bits, |s| < 4: its sum is exact, and the mean is off by two roundings, d = s - mean by at
    most 2^-21 and by whole units of s's last bit.  C d is exact again, and what is left of d after its own mean is taken off is
    two roundings of it, 2^-44; times eps^-1/2 = 1,000 and |gamma| < 16, y - beta is below 2^-30 but for y's own rounding."""
    values = torch.tensor([3.5, -1.0, 0.15625, 2.984375, -0.0])
    _, _, gamma, beta, _, _ = inputs(1, C, dtype, 9, False)
    x = values[:, None].expand(-1, C).contiguous().to(TORCH[dtype])
    Y = torch.full((len(values), C), float("nan"), device=DEV).to(TORCH[dtype])
    B.dsattn_layernorm(len(values), C, x.to(DEV), Y, gamma=gamma.to(DEV), beta=beta.to(DEV), io_dtype=CODE[dtype], eps=1e-6)
    torch.cuda.synchronize()
    assert gamma.abs().max() < 16
    step = half_step(dtype) * beta.abs() + (2.0 ** -24 * (beta.abs() + 2.0 ** -30) + 2.0 ** -30)
    assert ((Y.cpu().float() - beta).abs() <= step).all()


@pytest.mark.gpu
@pytest.mark.parametrize("C", [24, 64, 320, 1280, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_equal_numbers_infinities_and_nan(C, dtype):
    rows = 6
    x, _, gamma, beta, dy, _ = inputs(rows, C, dtype, 5, False)
    x[0] = 3.5
    x[2, C // 2] = float("inf")
    x[4, C - 1] = float("nan")
    for out in (dtype, "e4m3"):
        Y = torch.zeros(rows, C, device=DEV).to(TORCH[out])
        scales = torch.zeros(rows, device=DEV) if out == "e4m3" else None
        B.dsattn_layernorm(rows, C, x.to(DEV), Y, gamma=gamma.to(DEV), beta=beta.to(DEV), scales=scales, io_dtype=CODE[dtype],
                           out_dtype=CODE[out])
        torch.cuda.synchronize()
        y = Y.cpu().float()
        assert y[2].isnan().all() and y[4].isnan().all()
        if out == "e4m3":
            assert scales[2].isnan() and scales[4].isnan()
        else:
            assert (y[0] == beta.to(TORCH[dtype]).float()).all()
        keep = [1, 3, 5]
        check(dtype, out, x[keep], None, gamma, beta, 1e-6, None, Y[keep], None if scales is None else scales[keep])
    dX = torch.zeros(rows, C, device=DEV).to(TORCH[dtype])
    B.dsattn_layernorm_backward(rows, C, x.to(DEV), dy.to(DEV), dX, gamma=gamma.to(DEV), io_dtype=CODE[dtype])
    torch.cuda.synchronize()
    got = dX.cpu().float()
    assert got[2].isnan().all() and got[4].isnan().all() and got[0].isfinite().all()
    near(got[keep], gradients(x[keep], None, gamma, 1e-6, dy[keep], None)[0], half_step(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("C", [40, 1280, 20000])
def test_rows_beyond_the_range_of_their_squares(C):
    """Rows of 2^-60, 2^90 and 2^120 times an ordinary one give its result, eps 0."""
    x, _, gamma, beta, dy, _ = inputs(1, C, "f32", 6, False)
    x = x / x.abs().max()
    power = torch.tensor([1.0, 2.0 ** -60, 2.0 ** -110, 2.0 ** 90, 2.0 ** 120])
    xs, dys = x * power[:, None], dy.expand(5, C).contiguous()
    Y, dX = torch.empty(5, C, device=DEV), torch.empty(5, C, device=DEV)
    dg, db = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    B.dsattn_layernorm(5, C, xs.to(DEV), Y, gamma=gamma.to(DEV), beta=beta.to(DEV), io_dtype=B.DSATTN_F32, eps=0.0)
    B.dsattn_layernorm_backward(5, C, xs.to(DEV), dys.to(DEV), dX, gamma=gamma.to(DEV), dgamma=dg, dbeta=db,
                                workspace=space(5, C, "f32"), io_dtype=B.DSATTN_F32, eps=0.0)
    torch.cuda.synchronize()
    # (2^-110: a number of the row may be below 2^-126, and is off by half of 2^-149 then, 2^-40 of the largest)
    check("f32", "f32", x.expand(5, C), None, gamma, beta, 0.0, None, Y)
    want, tol = gradients(x.expand(5, C), None, gamma, 0.0, dys, None)[0]
    p = power.double()[:, None]
    near(dX.cpu().double() * p, (want, tol + 2.0 ** -149 * p))


@pytest.mark.gpu
@pytest.mark.parametrize("C,mean", [(320, 1000.0), (1280, 300.0), (20000, 1000.0)])
def test_rows_far_from_zero(C, mean):
    """A mean of hundreds of deviations costs the differences nothing but the rounding of s itself."""
    run(9, C, "f32", "f32", 12, residual=False, mean=mean)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,C", [(5000, 320), (40, 1280), (300, 20000), (3, 7)])
def test_the_same_call_gives_the_same_bits_and_rows_stand_alone(rows, C):
    d, dX, dg, db = run_back(rows, C, "bf16", 21)
    other, og, ob = torch.empty_like(dX), torch.empty_like(dg), torch.empty_like(db)
    for _ in range(3):
        B.dsattn_layernorm_backward(rows, C, d["x"], d["dy"], other, residual=d["r"], gamma=d["g"], dsum=d["ds"], dgamma=og,
                                    dbeta=ob, workspace=space(rows, C, "bf16"))
        assert torch.equal(other, dX) and torch.equal(og, dg) and torch.equal(ob, db)
    one = torch.empty(1, C, device=DEV, dtype=torch.bfloat16)
    at = rows // 2
    own = {k: d[k][at:at + 1].clone() for k in ("x", "r", "dy", "ds")}  # (a row's place is not aligned in every shape)
    B.dsattn_layernorm_backward(1, C, own["x"], own["dy"], one, residual=own["r"], gamma=d["g"], dsum=own["ds"])
    assert torch.equal(one[0], dX[at])


def test_the_formula_against_differences():
    """In 64 bits: central differences of y . dy + s . ds, whose error is h^2 times third derivatives (h = 1e-4: 1e-7)."""
    g = torch.Generator().manual_seed(1)
    rows, C, h = 3, 11, 1e-4
    x, dy, ds = (torch.randn(rows, C, generator=g, dtype=torch.float64) for _ in range(3))
    gamma, beta = (torch.randn(C, generator=g, dtype=torch.float64) for _ in range(2))

    def loss(x, gamma, beta):
        _, _, n, _, _, _ = normed(x, None, 1e-6)
        return ((n * gamma + beta) * dy).sum() + (x * ds).sum()

    def differences(t, f):
        out = torch.zeros_like(t)
        for i in range(t.numel()):
            e = torch.zeros_like(t).view(-1)
            e[i] = h
            out.view(-1)[i] = (f(t + e.view_as(t)) - f(t - e.view_as(t))) / (2 * h)
        return out

    dx, dg, db = gradients(x, None, gamma, 1e-6, dy, ds)
    assert (differences(x, lambda t: loss(t, gamma, beta)) - dx[0]).abs().max() < 1e-6
    assert (differences(gamma, lambda t: loss(x, t, beta)) - dg[0]).abs().max() < 1e-6
    assert (differences(beta, lambda t: loss(x, gamma, t)) - db[0]).abs().max() < 1e-6


def _desc(**kw):
    d = dict(rows=4, channels=64, io_dtype=B.DSATTN_BF16, out_dtype=B.DSATTN_BF16, eps=1e-6)
    d.update(kw)
    return B.DsattnLnDesc(**d)


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(rows=-1), dict(rows=1 << 31), dict(channels=0), dict(channels=(1 << 20) + 1), dict(io_dtype=2),
    dict(io_dtype=3), dict(out_dtype=0), dict(io_dtype=0), dict(out_dtype=5), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf"))])
def test_bad_descriptors_are_refused(kw):
    lib, d, n = B.load(), _desc(**kw), ctypes.c_size_t()
    assert lib.dsattn_layernorm(ctypes.byref(d), 0x10000, None, None, None, None, 0x20000, None, None) == B.DSATTN_EINVAL
    assert lib.dsattn_layernorm_backward(ctypes.byref(d), 0x10000, None, None, 0x20000, None, 0x30000, None, None, None, 0,
                                         None) == B.DSATTN_EINVAL
    assert lib.dsattn_layernorm_backward_workspace(ctypes.byref(d), ctypes.byref(n)) == B.DSATTN_EINVAL
    assert B.dsattn_last_error()


def test_bad_pointers_are_refused():
    lib = B.load()
    d, e = ctypes.byref(_desc()), ctypes.byref(_desc(out_dtype=B.DSATTN_E4M3))
    n = 4 * 64 * 2
    bad = [(None, 0x10000, None, None, None, None, 0x20000, None), (d, None, None, None, None, None, 0x20000, None),
           (d, 0x10000, None, None, None, None, None, None), (d, 0x10008, None, None, None, None, 0x20000, None),
           (d, 0x10000, None, None, 0x30004, None, 0x20000, None), (d, 0x10000, None, None, None, None, 0x20000, 0x40000),
           (e, 0x10000, None, None, None, None, 0x20000, None), (e, 0x10000, None, None, None, None, 0x20000, 0x40002),
           (d, 0x10000, None, None, None, None, 0x10010, None), (d, 0x10000, 0x30000, None, None, 0x30000 + n - 16, 0x20000, None),
           (d, 0x10000, None, None, None, 0x20000, 0x20000, None), (e, 0x10000, None, None, None, None, 0x10000, 0x40000),
           (d, 0x10000, None, None, 0x20000, None, 0x20000, None), (e, 0x10000, None, None, None, None, 0x20000, 0x10000)]
    for args in bad:
        assert lib.dsattn_layernorm(*args, None) == B.DSATTN_EINVAL, args
    size = B.dsattn_layernorm_backward_workspace(4, 64)
    assert size > 0
    long = ctypes.byref(_desc(channels=20000))
    bad = [(None, 0x10000, None, None, 0x20000, None, 0x30000, None, None, None, 0),
           (d, None, None, None, 0x20000, None, 0x30000, None, None, None, 0),
           (d, 0x10000, None, None, None, None, 0x30000, None, None, None, 0),
           (d, 0x10000, None, None, 0x20000, None, None, None, None, None, 0),
           (e, 0x10000, None, None, 0x20000, None, 0x30000, None, None, None, 0),          # gradients in 8 bits
           (d, 0x10008, None, None, 0x20000, None, 0x30000, None, None, None, 0),
           (d, 0x10000, None, None, 0x20000, 0x40008, 0x30000, None, None, None, 0),
           (d, 0x10000, None, None, 0x20000, None, 0x30000, 0x50002, None, 0x60000, size),
           (d, 0x10000, None, None, 0x20000, None, 0x30000, 0x50000, None, None, size),    # sums without a workspace
           (d, 0x10000, None, None, 0x20000, None, 0x30000, 0x50000, None, 0x60000, size - 1),
           (d, 0x10000, None, None, 0x20000, None, 0x30000, 0x50000, None, 0x60008, size),
           (d, 0x10000, None, None, 0x20000, None, 0x20010, None, None, None, 0),          # dX half over dY
           (d, 0x10000, None, 0x30000, 0x20000, None, 0x30000, None, None, None, 0),       # dX over gamma
           (d, 0x10000, None, None, 0x20000, None, 0x30000, 0x50000, 0x50000, 0x60000, size),
           (d, 0x10000, None, None, 0x20000, None, 0x30000, 0x50000, None, 0x10000, size),  # workspace over X
           (long, 0x100000, None, None, 0x200000, None, 0x200000, 0x500000, None, 0x600000, 1 << 30)]  # in place, long rows
    for args in bad:
        assert lib.dsattn_layernorm_backward(*args, None) == B.DSATTN_EINVAL, args


def test_launches_that_are_too_large_are_refused():
    """At addresses that no tensor has, so that nothing else is wrong with the calls; nothing runs."""
    lib, p = B.load(), [k << 50 for k in range(1, 8)]
    d = _desc(rows=1 << 24, channels=4096)  # 256 threads a row
    assert lib.dsattn_layernorm(ctypes.byref(d), p[0], None, None, None, None, p[1], None, None) == B.DSATTN_EUNSUPPORTED
    d = _desc(rows=1 << 24, channels=65536)
    assert lib.dsattn_layernorm(ctypes.byref(d), p[0], None, None, None, None, p[1], None, None) == B.DSATTN_EUNSUPPORTED
    for rows, sums in ((1 << 24, False), (64 * 65535 + 1, True)):
        need = B.dsattn_layernorm_backward_workspace(rows, 20000)
        assert lib.dsattn_layernorm_backward(ctypes.byref(_desc(rows=rows, channels=20000)), p[0], None, None, p[1], None, p[2],
                                             p[3] if sums else None, None, p[4] if sums else None, need, None) == B.DSATTN_EUNSUPPORTED


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    x = torch.zeros(4, 64, device=DEV, dtype=torch.bfloat16)
    w = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    for bad in (x[:3], x.float(), x.cpu(), torch.zeros(4, 128, device=DEV, dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError):
            B.dsattn_layernorm(4, 64, x, bad)
        with pytest.raises(ValueError):
            B.dsattn_layernorm_backward(4, 64, x, bad, x.clone())
    c = torch.zeros(64, device=DEV)
    with pytest.raises(ValueError):
        B.dsattn_layernorm_backward(4, 64, x, x, x.clone(), dgamma=c, workspace=w.float())
    with pytest.raises(ValueError):
        B.dsattn_layernorm_backward(4, 64, x, x, x.clone(), dgamma=c.bfloat16(), workspace=w)
    with pytest.raises(B.DsattnError):
        B.dsattn_layernorm_backward(4, 64, x, x, x.clone(), dgamma=c, workspace=w[:16])
