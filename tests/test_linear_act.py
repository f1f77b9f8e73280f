"""dsattn_linear_act: refusals on the host, and parity with the formula in 64 bits.

Tolerances: z is a sum of n = c_in products in fp32, off by at most n u times the sum of the products'
sizes (u = 2^-23: the matrix instructions may cut where they do not round), and three roundings of
scales and bias.  The activations have slopes of at most 1.13 and are evaluated to within 2^-20 of
their argument's size; the gate's product, the residual and the output add half a step each.  The matrix
instructions on 8 bits drop what is more than 13 bits below the largest product of a group (measured on the
instructions: 2^14 + 2^1 is kept, 2^14 + 2^0 is not), which a bf16 output is given: 2^-13 of the largest product
for each of a group's 64 channels.  An fp32 output has fp32 sums of them."""
import ctypes
import math

import pytest
import torch

from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
CODE = {"f32": B.DSATTN_F32, "bf16": B.DSATTN_BF16, "e4m3": B.DSATTN_E4M3}
ACTS = {"none": B.DSATTN_ACT_NONE, "relu": B.DSATTN_ACT_RELU, "gelu": B.DSATTN_ACT_GELU,
        "gelu_tanh": B.DSATTN_ACT_GELU_TANH, "silu": B.DSATTN_ACT_SILU}


def activate(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return z / 2 * torch.special.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def inputs(M, K, N, dtype, out, seed, gated, bias, residual, scaled):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def rand(*s):
        return torch.randn(*s, generator=g, device=DEV)

    sets = 2 if gated else 1
    x, w = rand(M, K), [rand(N, K) * K ** -0.5 for _ in range(sets)]
    sx = sw = None
    if dtype == "e4m3":
        x, w = x * 16, [a * 100 for a in w]
        if scaled:
            sx, sw = torch.exp(0.5 * rand(M)) / 16, [torch.exp(0.3 * rand(N)) / 100 for _ in range(sets)]
        else:
            w = [a / 1600 * 16 for a in w]
    return {"X": x.to(TORCH[dtype]), "W": [a.to(TORCH[dtype]) for a in w], "sx": sx, "sw": sw,
            "b": [rand(N), None][:sets] if bias == "first" else [rand(N) for _ in range(sets)] if bias else None,
            "R": rand(M, N).to(TORCH[out]) if residual else None}


def reference(t, act, out):
    """(y, tolerance) in 64 bits."""
    x = t["X"].double()
    z, e = [], []
    for k, w in enumerate(t["W"]):
        w = w.double()
        y, size = x @ w.t(), x.abs() @ w.abs().t()
        if t["sx"] is not None:
            s = t["sx"].double()[:, None] * t["sw"][k].double()
            y, size = y * s, size * s
        if t["b"] is not None and t["b"][k] is not None:
            y, size = y + t["b"][k].double(), size + t["b"][k].double().abs()
        z.append(y)
        err = size * (x.shape[1] + 4) * 2.0 ** -23
        if t["X"].dtype == torch.float8_e4m3fn and out == "bf16":
            err = err + cut(x, w) * (1.0 if t["sx"] is None else s)
        e.append(err)
    y, tol = activate(z[0], act), 1.13 * e[0] + 2.0 ** -20 * z[0].abs()
    if len(z) == 2:
        tol = tol * (z[1].abs() + e[1]) + y.abs() * e[1] + 2.0 ** -24 * (y * z[1]).abs()
        y = y * z[1]
    if t["R"] is not None:
        y = y + t["R"].double()
        tol = tol + 2.0 ** -24 * y.abs()
    half = torch.finfo(TORCH[out]).eps / 2
    return y, tol * (1 + half) + half * y.abs()


def cut(x, w):
    """64 2^-13 max|x| max|w| of every 64 channels, summed."""
    top = [torch.nn.functional.pad(a.abs().nan_to_num(0.0, 0.0), (0, -a.shape[1] % 64)).reshape(a.shape[0], -1, 64).amax(-1)
           for a in (x, w)]
    return 64 * 2.0 ** -13 * top[0] @ top[1].t()


def call(t, M, K, N, dtype, out, act, Y, flags=0, residual="R"):
    B.dsattn_linear_act(M, K, N, t["X"], t["W"], Y, biases=t["b"], residual=t[residual] if residual == "R" else residual,
                        x_scales=t["sx"], w_scales=t["sw"], act=ACTS[act], io_dtype=CODE[dtype], out_dtype=CODE[out],
                        flags=flags)


def run(M, K, N, dtype, out, act="none", gated=False, bias=True, residual=False, scaled=True, flags=0, seed=1):
    t = inputs(M, K, N, dtype, out, seed + M + K + N, gated, bias, residual, scaled)
    guard = torch.full((M * N + 64,), 12345.0, device=DEV).to(TORCH[out])
    Y = guard[:M * N].view(M, N)
    print(f"[case] linear_act {M} x {K} x {N} {dtype} -> {out} {act} gated {gated} bias {bias} residual {residual} "
          f"scaled {scaled} flags {flags}", flush=True)
    call(t, M, K, N, dtype, out, act, Y, flags)
    torch.cuda.synchronize()
    y, tol = reference(t, act, out)
    off = (Y.double() - y).abs()
    assert (off <= tol).all(), f"{(off / tol).max().item()} of the tolerance"
    assert (guard[M * N:].float() == guard[-1].float()).all(), "written past the end"
    return t, Y


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("e4m3", "bf16"), ("e4m3", "f32")]
SIZES = [(1, 1, 1), (1, 16, 8), (1, 320, 1280), (2, 7, 3), (3, 24, 40), (5, 160, 17), (16, 64, 64), (17, 136, 72), (33, 1280, 320),
         (64, 48, 200), (65, 320, 129), (100, 640, 96), (127, 256, 260), (160, 1280, 1280), (255, 80, 320), (257, 144, 514),
         (600, 72, 1000), (1030, 400, 136), (2000, 1280, 648), (4099, 320, 320)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_products(M, K, N, dtype, out):
    run(M, K, N, dtype, out, residual=M % 2 == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_gated_products(M, K, N, dtype, out):
    run(M, K, N, dtype, out, act="gelu", gated=True, residual=M % 2 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("bias,residual,scaled", [(False, False, True), (True, True, False), ("first", True, True)])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("M,K,N", [(3, 128, 72), (300, 192, 136)])
def test_epilogues(M, K, N, dtype, out, act, gated, bias, residual, scaled):
    run(M, K, N, dtype, out, act, gated, bias, residual, scaled)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("M,K,N,gated", [(9000, 640, 1280, False), (70000, 256, 320, False), (20000, 1024, 1032, False),
                                         (20000, 320, 512, True), (33333, 136, 776, True), (8192, 2560, 256, False)])
def test_large_products(M, K, N, gated, dtype, out):
    run(M, K, N, dtype, out, act="silu" if gated else "none", gated=gated, residual=not gated)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
def test_generic_kernel(dtype, out):
    run(77, 320, 130, dtype, out, act="gelu_tanh", gated=True, residual=True, flags=B.DSATTN_FLAG_FORCE_GENERIC)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("M,K,N", [(2, 320, 64), (200, 320, 200), (30000, 256, 512)])
def test_residual_in_place(M, K, N, dtype, out):
    t = inputs(M, K, N, dtype, out, 9, False, True, True, True)
    y, tol = reference(t, "silu", out)
    Y = t["R"].clone()
    call(t, M, K, N, dtype, out, "silu", Y, residual=Y)
    torch.cuda.synchronize()
    assert ((Y.double() - y).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("M,K,N", [(2, 320, 64), (200, 320, 200), (20000, 256, 512)])
def test_infinities_and_nan_stay_in_their_rows_and_channels(M, K, N, dtype, out):
    t = inputs(M, K, N, dtype, out, 4, False, True, False, True)
    t["X"][1, 5] = float("nan")
    if dtype != "e4m3":  # (e4m3 has no infinity)
        t["X"][0, 3] = float("inf")
    else:
        t["W"][0][N - 1, 2] = float("nan")
    Y = torch.empty(M, N, device=DEV, dtype=TORCH[out])
    call(t, M, K, N, dtype, out, "none", Y)
    torch.cuda.synchronize()
    y, tol = reference(t, "none", out)
    want, got = y.isnan() | y.isinf(), ~Y.double().isfinite()
    assert torch.equal(want, got) and got[1].all()
    assert ((Y.double() - y).abs() <= tol)[~want].all()


@pytest.mark.gpu
def test_two_calls_give_the_same_bits():
    for M, K, N, dtype, out in ((1, 1280, 1280, "bf16", "bf16"), (40, 5120, 64, "bf16", "f32"), (160, 1280, 1280, "e4m3", "bf16"),
                                (20000, 640, 640, "bf16", "bf16")):
        t = inputs(M, K, N, dtype, out, 8, False, True, False, True)
        got = []
        for _ in range(2):
            Y = torch.empty(M, N, device=DEV, dtype=TORCH[out])
            call(t, M, K, N, dtype, out, "none", Y)
            got.append(Y)
        torch.cuda.synchronize()
        assert torch.equal(got[0].view(torch.uint8), got[1].view(torch.uint8))


def _desc(**kw):
    d = dict(rows=4, c_in=64, c_out=32, n_w=1, act=0, io_dtype=B.DSATTN_BF16, out_dtype=B.DSATTN_BF16, flags=0)
    d.update(kw)
    return B.DsattnLinearActDesc(**d)


def _vps(*p):
    return (ctypes.c_void_p * len(p))(*p)


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(rows=1 << 31), dict(c_in=0), dict(c_out=0), dict(n_w=0), dict(n_w=3), dict(act=-1), dict(act=5),
    dict(io_dtype=3), dict(out_dtype=2), dict(io_dtype=0), dict(flags=2), dict(flags=8)])
def test_bad_descriptors_are_refused(kw):
    rc = B.load().dsattn_linear_act(ctypes.byref(_desc(**kw)), 0x10000, None, _vps(0x20000, 0x30000), None, None, None,
                                    0x40000, None)
    assert rc == B.DSATTN_EINVAL and B.dsattn_last_error()


def test_bad_pointers_are_refused():
    lib = B.load()
    d, g = ctypes.byref(_desc()), ctypes.byref(_desc(n_w=2))
    e = ctypes.byref(_desc(io_dtype=B.DSATTN_E4M3))
    W = _vps(0x20000)
    bad = [(None, 0x10000, None, W, None, None, None, 0x40000), (d, None, None, W, None, None, None, 0x40000),
           (d, 0x10000, None, None, None, None, None, 0x40000), (d, 0x10000, None, _vps(None), None, None, None, 0x40000),
           (d, 0x10000, None, W, None, None, None, None), (d, 0x10004, None, W, None, None, None, 0x40000),
           (d, 0x10000, None, _vps(0x20008), None, None, None, 0x40000), (d, 0x10000, None, W, None, None, None, 0x40002),
           (d, 0x10000, None, W, None, _vps(0x50002), None, 0x40000), (d, 0x10000, None, W, None, None, 0x60008, 0x40000),
           (d, 0x10000, 0x50000, W, None, None, None, 0x40000),             # scales of 16-bit operands
           (d, 0x10000, None, W, _vps(0x50000), None, None, 0x40000),
           (e, 0x10000, 0x50002, W, None, None, None, 0x40000), (e, 0x10000, None, W, _vps(0x50001), None, None, 0x40000),
           (d, 0x10000, None, W, None, None, None, 0x10000),                # Y over X
           (d, 0x10000, None, W, None, None, None, 0x20010),                # Y over W
           (g, 0x10000, None, _vps(0x20000, 0x40000), None, None, None, 0x40000),
           (d, 0x10000, None, W, None, None, 0x40010, 0x40000),             # half over the residual
           (d, 0x10000, None, W, None, _vps(0x40000), None, 0x40000),       # Y over the bias
           (e, 0x10000, 0x40000, W, None, None, None, 0x40000)]             # Y over the scales
    for args in bad:
        assert lib.dsattn_linear_act(*args, None) == B.DSATTN_EINVAL, args


def test_binding_checks_tensors():
    x, w, y = (torch.zeros(*s, dtype=torch.bfloat16) for s in ((4, 64), (32, 64), (4, 32)))
    b = torch.zeros(32)
    for kw in (dict(X=x[:3]), dict(X=x.float()), dict(Ws=[w[:31]]), dict(Ws=[w, w.float()]), dict(Y=y.float()),
               dict(biases=[b[:31]]), dict(biases=[b.double()]), dict(residual=x), dict(x_scales=b), dict(Ws=[]),
               dict(Ws=[w, w, w]), dict(biases=[b, b]), dict(w_scales=[b, b]), dict(Ws=[w.t()]), {}):
        args = {"X": x, "Ws": [w], "Y": y, **kw}
        with pytest.raises(ValueError, match="dsattn_linear_act"):
            B.dsattn_linear_act(4, 64, 32, **args)
