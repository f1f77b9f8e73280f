"""dsattn_linear_act_backward: refusals on the host, the formula against differences, and parity with it in 64 bits.

Tolerances: z is off by (c_in + 4) 2^-23 times the sum of its products' sizes (the matrix instructions may cut where they do not
round).  The activations' slopes are at most 1.13 and change by at most 1.13 a unit; both are evaluated to within 2^-20
of 1 + |z|.  dz takes that, and three roundings; where a product takes it in bf16, half a step more.  dX and dW are sums of n
products, n 2^-23 of their sizes, of numbers that are off by that much, and are rounded once; dbias is a sum of fp32
numbers.  Where relu's slope jumps within z's error dy is 0."""
import ctypes
import math

import pytest
import torch

import test_linear_act as L
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
TORCH, CODE, ACTS = L.TORCH, L.CODE, L.ACTS


def slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return (1 + t) / 2 + z / 2 * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * torch.sigmoid(-z)
    return torch.ones_like(z)


def inputs(M, K, N, dtype, act, seed, gated, bias):
    t = L.inputs(M, K, N, dtype, dtype, seed, gated, bias, False, False)
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    t["dY"] = torch.randn(M, N, generator=g, device=DEV).to(TORCH[dtype])
    if act == "relu":
        z, e = products(t)
        t["dY"] = torch.where(z[0].abs() <= 2 * e[0], torch.zeros_like(t["dY"]), t["dY"])
    return t


def products(t):
    x, z, e = t["X"].double(), [], []
    for k, w in enumerate(t["W"]):
        w = w.double()
        y, size = x @ w.t(), x.abs() @ w.abs().t()
        if t["b"] is not None and t["b"][k] is not None:
            y, size = y + t["b"][k].double(), size + t["b"][k].double().abs()
        z.append(y)
        e.append(size * (x.shape[1] + 4) * 2.0 ** -23)
    return z, e


def reference(t, act):
    """dX, [dW], [dbias], each with its tolerance, in 64 bits."""
    x, dy = t["X"].double(), t["dY"].double()
    half = torch.finfo(t["X"].dtype).eps / 2
    z, e = products(t)
    y, d = L.activate(z[0], act), slope(z[0], act)
    if act == "none":
        ey, ed = e[0], torch.zeros_like(z[0])
    else:
        ey, ed = 1.13 * e[0] + 2.0 ** -20 * (1 + z[0].abs()), (0 if act == "relu" else 1.13) * e[0] + 2.0 ** -20 * (1 + z[0].abs())
    if len(z) == 2:
        dz = [dy * z[1] * d, dy * y]
        ez = [dy.abs() * ((z[1].abs() + e[1]) * ed + e[1] * d.abs()) + 3 * 2.0 ** -24 * dz[0].abs(), dy.abs() * ey + 2.0 ** -24 * dz[1].abs()]
    else:
        dz, ez = [dy * d], [dy.abs() * ed + 2.0 ** -24 * (dy * d).abs()]
    same = act == "none" and len(z) == 1
    if same:
        ez = [torch.zeros_like(dy)]
    db = [(v.sum(0), ev.sum(0) + v.abs().sum(0) * v.shape[0] * 2.0 ** -24) for v, ev in zip(dz, ez)]
    # the operand of the two products
    eo = ez if t["X"].dtype == torch.float32 or same else [ev * (1 + half) + half * v.abs() for v, ev in zip(dz, ez)]
    dx, ex = torch.zeros_like(x), torch.zeros_like(x)
    n = len(z) * dy.shape[1]
    for v, ev, w in zip(dz, eo, t["W"]):
        w = w.double()
        dx, ex = dx + v @ w, ex + ev @ w.abs() + (n + 4) * 2.0 ** -23 * ((v.abs() + ev) @ w.abs())
    dw = [(v.t() @ x, ev.t() @ x.abs() + (len(x) + 4) * 2.0 ** -23 * ((v.abs() + ev).t() @ x.abs())) for v, ev in zip(dz, eo)]

    def rounded(v, tol):
        return v, tol * (1 + half) + half * v.abs()

    return rounded(dx, ex), [rounded(*p) for p in dw], db


def near(got, want, what):
    off = (got.double() - want[0]).abs()
    assert (off <= want[1]).all(), f"{what}: {(off / want[1].clamp_min(1e-300)).max().item()} of the tolerance"


def space(M, K, N, dtype, act, gated, flags=0):
    n = B.dsattn_linear_act_backward_workspace(M, K, N, n_w=2 if gated else 1, act=ACTS[act], io_dtype=CODE[dtype], flags=flags)
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None  # (NaN, read before written)


def call(t, M, K, N, dtype, act, dX, dW, db, flags=0, ws="own"):
    B.dsattn_linear_act_backward(M, K, N, t["X"], t["W"], t["dY"], dX=dX, dWs=dW, dbiases=db, biases=t["b"], act=ACTS[act],
                                 workspace=space(M, K, N, dtype, act, len(t["W"]) == 2, flags) if ws == "own" else ws,
                                 io_dtype=CODE[dtype], flags=flags)


def guarded(n, dtype):
    g = torch.full((n + 64,), 7.0, device=DEV).to(dtype)
    return g, g[:n]


def run(M, K, N, dtype, act="none", gated=False, bias=True, want="xwb", flags=0, seed=1):
    t = inputs(M, K, N, dtype, act, seed + M + K + N, gated, bias)
    sets = len(t["W"])
    tt = TORCH[dtype]
    gx, dX = guarded(M * K, tt)
    gw = [guarded(N * K, tt) for _ in range(sets)]
    gb = [guarded(N, torch.float32) for _ in range(sets)]
    dX = dX.view(M, K) if "x" in want else None
    dW = [g[1].view(N, K) for g in gw] if "w" in want else None
    db = [g[1] for g in gb] if "b" in want else None
    if want == "second":
        dW, db = [None, gw[1][1].view(N, K)], [gb[0][1], None]
    print(f"[case] linear_act_backward {M} x {K} x {N} {dtype} {act} gated {gated} bias {bias} want {want} flags {flags}", flush=True)
    call(t, M, K, N, dtype, act, dX, dW, db, flags)
    torch.cuda.synchronize()
    rx, rw, rb = reference(t, act)
    if dX is not None:
        near(dX, rx, "dX")
    for k in range(sets):
        if dW is not None and dW[k] is not None:
            near(dW[k], rw[k], f"dW[{k}]")
        if db is not None and db[k] is not None:
            near(db[k], rb[k], f"dbias[{k}]")
    for g in [gx] + [p[0] for p in gw + gb]:
        assert (g[-64:] == 7.0).all(), "written past the end"
    return t, dX, dW, db


SIZES = [(1, 8, 8), (1, 64, 320), (2, 320, 8), (17, 40, 24), (63, 72, 136), (64, 64, 64), (65, 128, 200), (130, 320, 264), (160, 264, 520),
         (257, 520, 72), (300, 1280, 640), (1000, 96, 320), (2050, 320, 328)]
ODD = [(1, 1, 1), (3, 5, 7), (33, 31, 8), (20, 8, 9), (129, 65, 130)]


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(65, 128, 200), (160, 264, 520), (3, 5, 7)])
def test_activations(M, K, N, dtype, act, gated):
    run(M, K, N, dtype, act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("none", False), ("gelu", True), ("silu", False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES + ODD)
def test_sizes(M, K, N, dtype, act, gated):
    run(M, K, N, dtype, act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("none", False), ("gelu", True), ("gelu_tanh", False), ("none", True)])
@pytest.mark.parametrize("M,K,N", [(4100, 640, 1288), (9000, 328, 640), (12345, 1280, 320), (700, 2560, 2568)])
def test_large_sizes(M, K, N, act, gated):
    run(M, K, N, "bf16", act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("none", False), ("gelu", True), ("silu", False)])
@pytest.mark.parametrize("M,K,N", [(500, 1288, 1304), (350, 2056, 1096), (1100, 1032, 1048), (2500, 1288, 1272), (130, 4104, 2056)])
def test_some_hundred_long_rows(M, K, N, act, gated):
    """Stages that are asked for two ahead, tiles down the columns, ends within a stage and a tile."""
    run(M, K, N, "bf16", act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("none", False), ("gelu", True), ("silu", False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 8, 5120), (1, 392, 5040), (33, 72, 4040), (100, 136, 3208), (160, 264, 2568)])
def test_few_rows_of_many_channels(M, K, N, dtype, act, gated):
    """dX's contraction split over workgroups, the last split a part of one."""
    run(M, K, N, dtype, act, gated)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(4100, 320, 648), (700, 1288, 640)])
def test_large_sizes_in_fp32(M, K, N):
    run(M, K, N, "f32", "gelu", True)
    run(M, K, N, "f32", "none", False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,gated", [("none", False), ("silu", True)])
@pytest.mark.parametrize("want", ["x", "w", "b", "xw", "xb", "wb"])
@pytest.mark.parametrize("M,K,N", [(130, 96, 72), (33, 31, 9)])
def test_some_outputs_only(M, K, N, dtype, act, gated, want):
    run(M, K, N, dtype, act, gated, want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [False, "first"])
@pytest.mark.parametrize("M,K,N", [(130, 96, 72), (33, 31, 9)])
def test_some_biases_and_some_sets_only(M, K, N, dtype, bias):
    run(M, K, N, dtype, "gelu", True, bias=bias)
    run(M, K, N, dtype, "gelu", True, bias=bias, want="second")


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("none", False), ("gelu", True)])
@pytest.mark.parametrize("M,K,N", [(130, 96, 72), (1000, 320, 640)])
def test_the_vector_kernels(M, K, N, act, gated):
    for dtype in ("f32", "bf16"):
        run(M, K, N, dtype, act, gated, flags=B.DSATTN_FLAG_FORCE_GENERIC)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(130, 96, 72), (5000, 320, 640), (33, 31, 9)])
def test_the_same_call_gives_the_same_bits(M, K, N):
    t, dX, dW, db = run(M, K, N, "bf16", "gelu", True)
    for _ in range(3):
        again = torch.empty_like(dX), [torch.empty_like(w) for w in dW], [torch.empty_like(b) for b in db]
        call(t, M, K, N, "bf16", "gelu", *again)
        assert torch.equal(again[0], dX) and all(map(torch.equal, again[1], dW)) and all(map(torch.equal, again[2], db))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_arguments_of_the_activations(dtype):
    """z of up to hundreds: slopes of 0 and 1, without NaN."""
    for act in ACTS:
        t = inputs(64, 8, 16, dtype, act, 5, True, True)
        t["W"] = [(w.float() * 100).to(TORCH[dtype]) for w in t["W"]]
        if act == "relu":
            z, e = products(t)
            t["dY"] = torch.where(z[0].abs() <= 2 * e[0], torch.zeros_like(t["dY"]), t["dY"])
        out = torch.empty_like(t["X"]), [torch.empty_like(w) for w in t["W"]], [torch.empty(16, device=DEV) for _ in range(2)]
        call(t, 64, 8, 16, dtype, act, *out)
        rx, rw, rb = reference(t, act)
        near(out[0], rx, act)
        for k in range(2):
            near(out[1][k], rw[k], act)
            near(out[2][k], rb[k], act)


def test_the_formula_against_differences():
    """In 64 bits: central differences of y . dy, whose error is h^2 times third derivatives (h = 1e-4: 1e-7)."""
    gen = torch.Generator().manual_seed(3)
    M, K, N, h = 3, 4, 5, 1e-4
    for act in ACTS:
        for sets in (1, 2):
            x, dy = torch.randn(M, K, generator=gen, dtype=torch.float64), torch.randn(M, N, generator=gen, dtype=torch.float64)
            w = torch.randn(sets, N, K, generator=gen, dtype=torch.float64)
            b = torch.randn(sets, N, generator=gen, dtype=torch.float64)

            def loss(x, w, b):
                z = [x @ w[k].t() + b[k] for k in range(sets)]
                y = L.activate(z[0], act)
                return ((y * z[1] if sets == 2 else y) * dy).sum()

            def differences(t, f):
                out = torch.zeros_like(t)
                for i in range(t.numel()):
                    e = torch.zeros_like(t).view(-1)
                    e[i] = h
                    out.view(-1)[i] = (f(t + e.view_as(t)) - f(t - e.view_as(t))) / (2 * h)
                return out

            z = [x @ w[k].t() + b[k] for k in range(sets)]
            assert z[0].abs().min() > 10 * h
            rx, rw, rb = reference({"X": x, "W": list(w), "b": list(b), "dY": dy}, act)
            assert (differences(x, lambda t: loss(t, w, b)) - rx[0]).abs().max() < 1e-5
            assert (differences(w, lambda t: loss(x, t, b)) - torch.stack([v[0] for v in rw])).abs().max() < 1e-5
            assert (differences(b, lambda t: loss(x, w, t)) - torch.stack([v[0] for v in rb])).abs().max() < 1e-5


def _desc(**kw):
    d = dict(rows=4, c_in=64, c_out=32, n_w=2, act=2, io_dtype=B.DSATTN_BF16, out_dtype=B.DSATTN_BF16, flags=0)
    d.update(kw)
    return B.DsattnLinearActDesc(**d)


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(rows=1 << 31), dict(c_in=0), dict(c_out=-1), dict(n_w=0), dict(n_w=3), dict(act=5), dict(act=-1),
    dict(io_dtype=2), dict(io_dtype=0), dict(out_dtype=0), dict(out_dtype=2), dict(flags=2), dict(flags=16),
    dict(rows=0x7fffffff, c_in=0x7fffffff), dict(c_in=0x7fffffff, c_out=0x7fffffff)])
def test_bad_descriptors_are_refused(kw):
    lib, d, n = B.load(), _desc(**kw), ctypes.c_size_t()
    w = (ctypes.c_void_p * 2)(0x200000, 0x300000)
    assert lib.dsattn_linear_act_backward(ctypes.byref(d), 0x100000, w, None, 0x400000, 0x500000, None, None, 0x600000, 1 << 40,
                                          None) == B.DSATTN_EINVAL
    assert lib.dsattn_linear_act_backward_workspace(ctypes.byref(d), ctypes.byref(n)) == B.DSATTN_EINVAL
    assert B.dsattn_last_error()


def test_bad_pointers_are_refused():
    lib, d = B.load(), ctypes.byref(_desc())
    need = B.dsattn_linear_act_backward_workspace(4, 64, 32, n_w=2, act=B.DSATTN_ACT_GELU)
    assert need > 0 and B.dsattn_linear_act_backward_workspace(4, 1, 1) == 0

    def two(a, b):
        return (ctypes.c_void_p * 2)(a, b)

    p = [0x1000000 * (k + 1) for k in range(9)]
    w, f = two(p[1], p[2]), lib.dsattn_linear_act_backward
    for args in [(None, p[0], w, None, p[3], p[4], None, None, p[5], need), (d, None, w, None, p[3], p[4], None, None, p[5], need),
                 (d, p[0], None, None, p[3], p[4], None, None, p[5], need), (d, p[0], w, None, None, p[4], None, None, p[5], need),
                 (d, p[0], two(p[1], None), None, p[3], p[4], None, None, p[5], need),
                 (d, p[0], two(p[1], p[2] + 8), None, p[3], p[4], None, None, p[5], need),
                 (d, p[0], w, two(p[6], p[7] + 2), p[3], p[4], None, None, p[5], need),
                 (d, p[0], w, None, p[3], p[4], two(p[6], p[7] + 4), None, p[5], need),
                 (d, p[0], w, None, p[3], p[4], None, two(p[6] + 2, None), p[5], need),
                 (d, p[0] + 4, w, None, p[3], p[4], None, None, p[5], need), (d, p[0], w, None, p[3], p[4], None, None, p[5] + 8, need),
                 (d, p[0], w, None, p[3], p[4], None, None, None, need), (d, p[0], w, None, p[3], p[4], None, None, p[5], need - 1),
                 (d, p[0], w, None, p[3], p[0], None, None, p[5], need), (d, p[0], w, None, p[3], p[3] + 16, None, None, p[5], need),
                 (d, p[0], w, None, p[3], p[4], two(p[1], None), None, p[5], need),
                 (d, p[0], w, None, p[3], p[4], two(p[6], p[6] + 16), None, p[5], need),
                 (d, p[0], w, None, p[3], p[4], None, two(p[5], None), p[5], need),
                 (d, p[0], w, None, p[3], p[4], None, None, p[0], need)]:
        assert f(*args, None) == B.DSATTN_EINVAL, args


def test_launches_that_are_too_large_are_refused():
    """At addresses that no tensor has, so that nothing else is wrong with the calls; nothing runs."""
    lib, p = B.load(), [k << 50 for k in range(1, 8)]
    for kw in (dict(rows=1 << 30, c_in=9, c_out=9, n_w=1, act=1), dict(rows=3, c_in=65537, c_out=65537, n_w=1, act=1),
               dict(rows=1 << 30, c_in=64, c_out=64, n_w=1, act=0, flags=B.DSATTN_FLAG_FORCE_GENERIC)):
        need = B.dsattn_linear_act_backward_workspace(kw["rows"], kw["c_in"], kw["c_out"], act=kw["act"], flags=kw.get("flags", 0))
        w = (ctypes.c_void_p * 2)(p[1], None)
        assert lib.dsattn_linear_act_backward(ctypes.byref(_desc(**kw)), p[0], w, None, p[2], p[3], None, None, p[4], need,
                                              None) == B.DSATTN_EUNSUPPORTED, kw


@pytest.mark.gpu
def test_tensors_that_do_not_fit_are_refused():
    bf = dict(dtype=torch.bfloat16, device=DEV)
    x, w, dy = torch.zeros(4, 64, **bf), torch.zeros(32, 64, **bf), torch.zeros(4, 32, **bf)
    for bad in (dy[:3], dy.float(), dy.cpu(), torch.zeros(4, 64, **bf)[:, ::2]):
        with pytest.raises(ValueError):
            B.dsattn_linear_act_backward(4, 64, 32, x, [w], bad, dX=torch.zeros_like(x))
    with pytest.raises(ValueError):
        B.dsattn_linear_act_backward(4, 64, 32, x, [w], dy, dWs=[w[:31].clone()])
    with pytest.raises(ValueError):
        B.dsattn_linear_act_backward(4, 64, 32, x, [w], dy, dWs=[w.clone(), w.clone()])
    with pytest.raises(ValueError):
        B.dsattn_linear_act_backward(4, 64, 32, x, [w, w, w], dy)
    with pytest.raises(ValueError):
        B.dsattn_linear_act_backward(4, 64, 32, x, [w], dy, dbiases=[dy])
