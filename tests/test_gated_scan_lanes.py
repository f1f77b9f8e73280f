"""dsattn_gated_scan and its backward pass at frames of many channels, against the formula: two channels a lane (bf16, from
65,536 channels of all streams on), eight bytes a lane in the forward pass (from 64 K lanes on), one where their number is odd;
streams alone, and what lies behind a workspace."""
import pytest
import torch

import test_gated_scan as R
from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
TWO = [("bf16", 1, 40, 160, 512), ("bf16", 2, 33, 81, 410), ("bf16", 1, 17, 129, 2050), ("bf16", 1, 1, 160, 1280)]
WIDE = [("bf16", 1, 35, 260, 1024), ("bf16", 2, 20, 131, 1004), ("f32", 1, 35, 130, 1024), ("f32", 3, 18, 60, 730), ("f32", 1, 1, 160, 1280)]
ONE = [("bf16", 1, 20, 81, 811), ("f32", 1, 20, 161, 815)]


@pytest.mark.gpu
@pytest.mark.parametrize("mode", list(R.MODES))
@pytest.mark.parametrize("dtype,Bs,T,P,C", TWO + WIDE + ONE)
def test_against_the_formula(Bs, T, P, C, dtype, mode):
    R.run(Bs, T, P, C, dtype, mode)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", list(R.MODES))
@pytest.mark.parametrize("dtype,T,P,C,counts", [
    ("bf16", 33, 81, 274, [33, 0, 16]), ("bf16", 20, 90, 1000, [17, 1, 20]), ("f32", 33, 45, 974, [0, 32, 5])])
def test_streams_of_different_lengths(T, P, C, counts, dtype, mode):
    R.run(len(counts), T, P, C, dtype, mode, counts)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,Bs,T,P,C", [("bf16", 2, 33, 81, 410), ("bf16", 2, 20, 131, 1004), ("f32", 3, 18, 60, 730)])
def test_in_place(Bs, T, P, C, dtype):
    shape, code = (Bs, T, P, C), R.CODE[dtype]
    t = [v.to(DEV) for v in R.inputs(*shape, dtype, 9)]
    Y, hT, S = torch.empty_like(t[0]), torch.empty_like(t[2]), torch.empty(Bs, -(-T // R.STEP), P, C, device=DEV)
    B.dsattn_gated_scan(*shape, t[0], t[1], Y, start_state=t[2], end_state=hT, states=S, io_dtype=code)
    for into in (0, 1):
        u = [v.clone() for v in t]
        B.dsattn_gated_scan(*shape, u[0], u[1], u[into], start_state=u[2], end_state=u[2], io_dtype=code)
        assert torch.equal(u[into], Y) and torch.equal(u[2], hT)
    dX, dG, dh = torch.empty_like(Y), torch.empty_like(Y), torch.empty_like(hT)
    B.dsattn_gated_scan_backward(*shape, t[0], t[1], S, t[3], dX, dG, dend_state=t[4], dstart_state=dh, io_dtype=code)
    for a, b in ((0, 1), (1, 0), (3, 1), (0, 3)):
        u = [v.clone() for v in t]
        B.dsattn_gated_scan_backward(*shape, u[0], u[1], S, u[3], u[a], u[b], dend_state=u[4], dstart_state=u[4], io_dtype=code)
        assert torch.equal(u[a], dX) and torch.equal(u[b], dG) and torch.equal(u[4], dh)


def both(shape, dtype, mode, t, counts, space):
    """Forward and backward pass with a workspace of its own: everything that they write."""
    x, g, h0, dy, dend = t
    Y, dX, dG = (torch.full_like(x, 7.0) for _ in range(3))
    hT, dh = torch.empty_like(h0), torch.empty_like(h0)
    S = torch.full((shape[0], -(-shape[1] // R.STEP), *shape[2:]), 7.0, device=DEV)
    kw = dict(mode=R.MODES[mode], counts=counts, workspace=space, io_dtype=R.CODE[dtype])
    B.dsattn_gated_scan(*shape, x, g, Y, start_state=h0, end_state=hT, states=S, **kw)
    B.dsattn_gated_scan_backward(*shape, x, g, S, dy, dX, dG, dend_state=dend, dstart_state=dh, **kw)
    torch.cuda.synchronize()
    return Y, hT, S, dX, dG, dh


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,mode", [("f32", "norm"), ("bf16", "mean"), ("bf16", "sum")])
@pytest.mark.parametrize("T,P,C,counts", [(1100, 1, 136, None), (1100, 1, 136, [1100, 700, 0]), (50, 9, 40, [50, 17, 1]), (33, 70, 320, None)])
def test_streams_stand_alone(T, P, C, counts, dtype, mode):
    """A stream of a batch gives the bits that it gives alone: these sizes are cut into the same chunks (of 32 frames and more), or are
    one, and a stream reads nothing of the others."""
    shape = (3, T, P, C)
    t = [v.to(DEV) for v in R.inputs(*shape, dtype, 8)]
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
    need, one = (B.dsattn_gated_scan_workspace(b, T, P, C, io_dtype=R.CODE[dtype]) for b in (3, 1))
    assert need == 3 * one
    got = both(shape, dtype, mode, t, cnt, R.space(*shape, dtype))
    for b in range(3):
        alone = both((1, T, P, C), dtype, mode, [v[b:b + 1].clone() for v in t], None if cnt is None else cnt[b:b + 1].clone(),
                     R.space(1, T, P, C, dtype))
        for name, x, y in zip(("Y", "hT", "S", "dX", "dG", "dh"), got, alone):
            assert torch.equal(x[b:b + 1], y), (b, name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Bs,T,P,C", [(1, 300, 1, 1), (2, 256, 1, 8), (3, 700, 1, 33), (1, 3000, 1, 24), (2, 2049, 1, 129), (1, 200, 9, 1000)])
def test_nothing_behind_the_workspace_is_written(Bs, T, P, C, dtype):
    shape, t = (Bs, T, P, C), [v.to(DEV) for v in R.inputs(Bs, T, P, C, dtype, 8)]
    need = B.dsattn_gated_scan_workspace(*shape, io_dtype=R.CODE[dtype])
    assert need
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    got = both(shape, dtype, "mean", t, None, room[:need])
    assert (room[need:] == 0xA5).all()
    for x, y in zip(got, both(shape, dtype, "mean", t, None, R.space(*shape, dtype))):
        assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Bs,T,P,C", [(1, 1, 1, 7), (2, 17, 3, 40), (1, 300, 1, 1), (3, 700, 1, 33), (1, 5000, 1, 24), (2, 2049, 1, 129),
                                      (1, 16384, 1, 1280), (5, 1587, 1, 432), (1, 200, 9, 1000), (1, 40, 160, 512), (2, 33, 81, 410), (1, 35, 260, 1024),
                                      (3, 18, 60, 730), (1, 130000, 1, 5)])
def test_whole_numbers_come_out_exact(Bs, T, P, C, dtype, counts):
    """Gates of 0 and 1 (infinite logits) and whole numbers: sums from one frame that begins anew to the next, without rounding but Y's and
    dX's own, however the frames are cut into chunks; dG is 0."""
    gen = torch.Generator().manual_seed(T + C)
    shape, dt = (Bs, T, P, C), R.TORCH[dtype]

    def whole(*s):
        return torch.randint(-9, 10, s, generator=gen).float()

    x, dy, h0, dend = whole(*shape), whole(*shape), whole(Bs, P, C), whole(Bs, P, C)
    keep = torch.rand(*shape, generator=gen) > 0.002
    g = torch.where(keep, float("inf"), float("-inf"))
    cnt = torch.randint(0, T + 1, (Bs,), generator=gen) if counts else torch.full((Bs,), T)
    t = [v.to(dt).to(DEV) for v in (x, g)] + [h0.to(DEV), dy.to(dt).to(DEV), dend.to(DEV)]
    got = both(shape, dtype, "sum", t, cnt.to(torch.int32).to(DEV) if counts else None, R.space(*shape, dtype))
    kd, xd, dd = keep.double().to(DEV), x.double().to(DEV), dy.double().to(DEV)

    def sums(v, at):
        """Sums of v along dimension 0 from the last one at or before each place at which `at` is 1, or from the start."""
        c = v.cumsum(0)
        from_ = torch.where(at.bool(), c - v, torch.full_like(c, -float("inf")))
        where = torch.where(at.bool(), torch.arange(len(v), device=DEV).view(-1, *[1] * (v.dim() - 1)), -1).cummax(0).values
        base = torch.gather(torch.where(from_.isinf(), 0.0, from_), 0, where.clamp_min(0))
        return c - torch.where(where < 0, 0.0, base)

    for b in range(Bs):
        n = int(cnt[b])
        v, anew = xd[b, :n].clone(), 1 - kd[b, :n]
        start = h0[b].double().to(DEV)
        h = sums(torch.cat([start[None], v]), torch.cat([torch.zeros_like(start)[None], anew]))  # h[t]: behind frame t - 1
        # from the end: what comes from behind a frame passes if the next one keeps
        end = dend[b].double().to(DEV)
        late = torch.cat([torch.zeros_like(end)[None], torch.zeros_like(end)[None], anew.flip(0)])[:n + 1]
        d = sums(torch.cat([end[None], dd[b, :n].flip(0)]), late).flip(0)  # d[n]: the end's gradient; d[t]: D_t
        for name, a, w, rest in (("Y", got[0], h[1:], 7.0), ("dX", got[3], d[:n], 7.0), ("dG", got[4], torch.zeros_like(v), 7.0)):
            assert torch.equal(a[b, :n], w.float().to(dt)), name
            assert (a[b, n:] == rest).all(), name
        assert torch.equal(got[1][b], h[-1].float())
        k = -(-n // R.STEP)
        assert torch.equal(got[2][b, :k], h[:-1:R.STEP].float() if n else h[:0].float()) and (got[2][b, k:] == 7.0).all()
        first = d[0] * kd[b, 0] if n else end
        assert torch.equal(got[5][b], first.float())
