"""dsattn_linear_act_backward at the sizes of its different kernels: some of the outputs only, and infinities and NaN, which reach the
rows and columns that their formula has them in and no others."""
import pytest
import torch

import test_linear_act_grad as G
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
SIZES = [(33, 72, 4040), (160, 264, 520), (350, 2056, 1096), (640, 640, 640), (1100, 1032, 1048), (4100, 640, 1288), (8200, 1032, 1288),
         (10000, 512, 2048)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,gated", [("none", False), ("silu", False), ("gelu", True)])
@pytest.mark.parametrize("want", ["x", "w", "b", "xw", "xb", "wb", "second"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_some_outputs_only(M, K, N, dtype, act, gated, want):
    if want == "second" and not gated:
        want = "xwb"
    G.run(M, K, N, dtype, act, gated, bias=want != "xw", want=want)


def gradients(t, M, K, N, dtype, act):
    out = torch.empty_like(t["X"]), [torch.empty_like(w) for w in t["W"]], [torch.empty(N, device=DEV) for _ in t["W"]]
    G.call(t, M, K, N, dtype, act, *out)
    torch.cuda.synchronize()
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,gated", [("none", False), ("silu", False), ("gelu", True)])
@pytest.mark.parametrize("M,K,N", [(1, 64, 72), (33, 31, 9), *SIZES])
def test_what_is_not_finite_stays_in_its_rows_and_columns(M, K, N, dtype, act, gated, bad):
    same = act == "none" and not gated
    for m, k, c in ((M - 1, K - 1, N - 1), (M // 2, K // 3, N // 2)):
        print(f"[case] {M} x {K} x {N} {dtype} {act} gated {gated}: {bad} at {m}, {k}, {c}", flush=True)
        rows, cols, ins = ([i for i in range(n) if i != at] for n, at in ((M, m), (N, c), (K, k)))
        # in dY: its row of dX, its channel of dW and dbias
        t = G.inputs(M, K, N, dtype, act, 5, gated, True)
        clean = gradients(t, M, K, N, dtype, act)
        t["dY"][m, c] = bad
        dX, dW, db = gradients(t, M, K, N, dtype, act)
        assert not dX[m].isfinite().any() and torch.equal(dX[rows], clean[0][rows])
        for s in range(len(dW)):
            assert not dW[s][c].isfinite().any() and torch.equal(dW[s][cols], clean[1][s][cols])
            assert not db[s][c].isfinite() and torch.equal(db[s][cols], clean[2][s][cols])
        # in X: its row of dX (but where dz is dY) and everything that is summed over rows, or its channel of dW alone
        t = G.inputs(M, K, N, dtype, act, 5, gated, True)
        t["X"][m, k] = bad
        dX, dW, db = gradients(t, M, K, N, dtype, act)
        assert torch.equal(dX[rows], clean[0][rows])
        if same:
            assert torch.equal(dX, clean[0]) and torch.equal(db[0], clean[2][0])
            assert not dW[0][:, k].isfinite().any() and torch.equal(dW[0][:, ins], clean[1][0][:, ins])
        # in a bias: its channel of dW and dbias; dX everywhere
        if not same:
            t = G.inputs(M, K, N, dtype, act, 5, gated, True)
            t["b"][0][c] = bad
            dX, dW, db = gradients(t, M, K, N, dtype, act)
            for s in range(len(dW)):
                assert torch.equal(dW[s][cols], clean[1][s][cols]) and torch.equal(db[s][cols], clean[2][s][cols])
            if bad != bad:
                assert dX.isnan().all() and all(w[c].isnan().all() and b[c].isnan() for w, b in zip(dW, db))
            elif not gated:  # a slope of 1, or of 0: dbias is dy's sum, or 0
                want = t["dY"][:, c].double().sum() if bad > 0 else torch.zeros((), device=DEV)
                assert (db[0][c].double() - want).abs() <= M * 2.0 ** -23 * t["dY"][:, c].double().abs().sum()
                assert dX.isfinite().all() and dW[0].isfinite().all()
