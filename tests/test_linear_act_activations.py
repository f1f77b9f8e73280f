"""The activations of dsattn_linear_act over all of their arguments, in every kernel.

An argument is put in by the bias, which is added in fp32 to a product of zeros, so that z is exact; what is left is
the activation's own error, half a step of the output's type, and nothing of the products."""
import math

import pytest
import torch

import test_linear_act as L
from paper_2406_16260_amd import binding as B
from test_linear_act_scales import sized

DEV = "cuda:0"


def arguments(n, act):
    """n numbers that an activation may be given: around zero, in its bend, in its tails, and far outside."""
    far = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3e38, 1e20, 5e9, -5e9, -1e20, -3e38, 1e-37, 60.0, -60.0, 9.0, -9.0, -5.5, -6.0])
    reach = 7.0 if act.startswith("gelu") else 60.0
    z = torch.linspace(-reach, reach, n - len(far) - 200)
    return torch.cat([far, z, torch.logspace(-12, 0, 100), -torch.logspace(-12, 0, 100)])


def allowed(z, act, vector):
    """How far act(z) may be off, in 64 bits: see the bounds' arithmetic."""
    one = torch.ones_like(z)
    if act == "none":
        return 0 * z
    if act == "relu":
        return 0 * z
    if act == "gelu":
        p = torch.special.ndtr(z)
        if vector:  # x / 2 (1 + erf(u)): erf off by 2 steps of 2^-24 and by its argument's 2^-23 u erf'(u) < 2^-24, the sum by 2^-24
            return z.abs() * 2.0 ** -23 + 2.0 ** -22 * (z * p).abs()
        # the fit, 2.93e-8 of P; its polynomial in fp32 moves the exponent by less than 2^-21 where P (1 - P) counts; exp2,
        # reciprocal and the last product are off by three steps of P
        return z.abs() * (2.93e-8 + 2.0 ** -21 * p * (1 - p) + 2.0 ** -22 * p)
    # x / (1 + e^-v), v rounded five times on the way: relative error |v| 2^-22 of e^-v, three steps of the rest
    v = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3) if act == "gelu_tanh" else z
    s = torch.sigmoid(v)
    rel = torch.minimum((v.abs() + 1) * 2.0 ** -22 * (1 - s), one) + 2.0 ** -21
    return (z * s).abs() * rel + 2.0 ** -120  # (below that e^-v is beyond fp32's range and the result zero)


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("act", sorted(L.ACTS))
def test_activations_over_their_arguments(act, out):
    for M, K, N, flags in sized("bf16", out):
        print(f"[case] {act} of {M} x {K} x {N} -> {out}, flags {flags}", flush=True)
        x, w = torch.zeros(M, K, device=DEV, dtype=torch.bfloat16), torch.zeros(N, K, device=DEV, dtype=torch.bfloat16)
        z = arguments(N, act).to(DEV)
        Y = torch.full((M, N), float("nan"), device=DEV, dtype=L.TORCH[out])
        B.dsattn_linear_act(M, K, N, x, [w], Y, biases=[z], act=L.ACTS[act], out_dtype=L.CODE[out], flags=flags)
        torch.cuda.synchronize()
        assert (Y == Y[0]).all()
        z = z.double()
        want = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)) if act == "gelu_tanh" else \
            z * torch.special.ndtr(z) if act == "gelu" else z * torch.sigmoid(z) if act == "silu" else L.activate(z, act)
        tol = allowed(z, act, flags != 0)
        half = torch.finfo(L.TORCH[out]).eps / 2
        off = (Y[0].double() - want).abs()
        over = off - (tol * (1 + half) + half * want.abs())
        at = over.argmax()
        assert (over <= 0).all(), (z[at].item(), want[at].item(), Y[0, at].item(), tol[at].item())
