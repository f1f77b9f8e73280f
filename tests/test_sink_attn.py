"""dsattn_sink_forward: refusals on the host, and parity with the definition in 64 bits.

Tolerances: a score is a sum of head_dim fp32 products, off by at most d = (head_dim + 4) 2^-23 |q| |k| scale
(Cauchy-Schwarz), and so is a weight, relatively, twice over (itself and the sum that it is divided by),
with 2^-20 for the exponential and the sums over the keys.  Weights of bf16 tensors may be rounded to bf16
for the product with V: 2^-8 each, in the numerator and in the denominator.  All of that times the weighted
mean of |v|; and half a step of the output's type."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2406_16260_amd import binding as B

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": B.DSATTN_F32, "bf16": B.DSATTN_BF16}


def slot(f, sinks, ring):
    return f if f < sinks else sinks + (f - sinks) % ring


class Stream:
    """Tensors of one call, and a history that fills the caches as calls before it would have."""

    def __init__(self, c, seed):
        self.c = c
        g = torch.Generator().manual_seed(seed)

        def rand(*s):
            return torch.randn(*s, generator=g).to(TORCH[c["dtype"]])

        Bn, T, P, h, hk, D = (c[k] for k in ("B", "T", "P", "h", "hk", "D"))
        self.start, self.counts = list(c["start"]), list(c["counts"])
        slots = c["sinks"] + c["ring"]
        self.Q, self.K, self.V = rand(Bn, T, P, h * D), rand(Bn, T, P, hk * D), rand(Bn, T, P, hk * D)
        # slots that no frame has been in hold NaN: nobody may look there
        self.Kc = torch.full((Bn, slots, P, hk * D), float("nan"), dtype=TORCH[c["dtype"]])
        self.Vc = self.Kc.clone()
        for b in range(Bn):
            for f in range(max(0, self.start[b] - c["ring"] - c["sinks"]), self.start[b]):
                self.put(b, f, rand(P, hk * D), rand(P, hk * D))
            for f in range(min(c["sinks"], self.start[b])):
                self.put(b, f, rand(P, hk * D), rand(P, hk * D))
            # rows behind the last new frame hold NaN too
            for t in (self.Q, self.K, self.V):
                t[b, self.counts[b]:] = float("nan")

    def put(self, b, f, k, v):
        s = slot(f, self.c["sinks"], self.c["ring"])
        self.Kc[b, s], self.Vc[b, s] = k, v

    def frame(self, b, f):
        t = f - self.start[b]
        if t >= 0:
            return self.K[b, t], self.V[b, t]
        s = slot(f, self.c["sinks"], self.c["ring"])
        return self.Kc[b, s], self.Vc[b, s]

    def reference(self, scale):
        """(O, tolerance) in 64 bits; rows behind the last new frame keep 777."""
        c = self.c
        Bn, T, P, h, hk, D = (c[k] for k in ("B", "T", "P", "h", "hk", "D"))
        O = torch.full((Bn, T, P, h, D), 777.0, dtype=torch.float64)
        tol = torch.zeros_like(O)
        half = torch.finfo(TORCH[c["dtype"]]).eps / 2
        weight = 2.0 ** -20 + (2 * 2.0 ** -8 if c["dtype"] == "bf16" else 0.0)
        for b in range(Bn):
            # all frames that a query of this call may see
            frames = [f for f in range(self.start[b] + self.counts[b])
                      if f < c["sinks"] or f >= self.start[b] - c["window"] + 1]
            if not frames or not self.counts[b]:
                O[b, :self.counts[b]] = 0
                continue
            kv = [self.frame(b, f) for f in frames]
            k = torch.stack([x for x, _ in kv]).double().reshape(-1, P, hk, D).repeat_interleave(h // hk, 2)
            v = torch.stack([x for _, x in kv]).double().reshape(-1, P, hk, D).repeat_interleave(h // hk, 2)
            q = self.Q[b, :self.counts[b]].double().reshape(-1, P, h, D)
            fr = torch.tensor(frames)[None, :]
            a = torch.arange(self.start[b], self.start[b] + self.counts[b])[:, None]
            seen = (fr <= a) & ((fr < c["sinks"]) | (a - fr < c["window"]))
            s = torch.einsum("tphd,jphd->phtj", q, k) * scale
            s = torch.where(seen, s, -float("inf"))
            top = s.amax(-1, keepdim=True)
            e = torch.where(seen, torch.exp(s - torch.where(top.isinf(), 0.0, top)), 0.0)
            total = e.sum(-1, keepdim=True)
            w = torch.where(total > 0, e / total, 0.0)
            o = torch.einsum("phtj,jphd->tphd", w, v)
            size = torch.einsum("phtj,jphd->tphd", w, v.abs())
            d = (D + 4) * 2.0 ** -23 * abs(scale) * q.norm(dim=-1).amax() * k.norm(dim=-1).amax()
            n = self.counts[b]
            O[b, :n] = o
            tol[b, :n] = (2 * d + weight) * size + half * o.abs()
        return O.reshape(Bn, T, P, h * D), tol.reshape(Bn, T, P, h * D) * (1 + 2.0 ** -6)

    def caches(self):
        Kc, Vc = self.Kc.clone(), self.Vc.clone()
        c = self.c
        for b in range(c["B"]):
            for t in range(self.counts[b]):
                s = slot(self.start[b] + t, c["sinks"], c["ring"])
                Kc[b, s], Vc[b, s] = self.K[b, t], self.V[b, t]
        return Kc, Vc


def space_for(c, flags=0):
    n = B.dsattn_sink_workspace(c["B"], c["T"], c["P"], c["h"], c["hk"], c["D"], c["sinks"], c["window"], c["ring"],
                                io_dtype=CODE[c["dtype"]], flags=flags)
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV)


def same_bits(a, b):
    a, b = a.cpu().contiguous(), b.cpu().contiguous()
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def case(dtype="bf16", B=1, T=1, P=1, h=1, hk=None, D=64, sinks=2, window=8, ring=None, start=0, counts=None):
    hk = h if hk is None else hk
    start = [start] * B if isinstance(start, int) else start
    return dict(dtype=dtype, B=B, T=T, P=P, h=h, hk=hk, D=D, sinks=sinks, window=window,
                ring=max(window, 1) if ring is None else ring, start=start,
                counts=[T] * B if counts is None else counts)


def forward(s, c, O, Kc, Vc, scale=0.0, flags=0, space=None):
    i32 = dict(dtype=torch.int32, device=DEV)
    B.dsattn_sink_forward(c["B"], c["T"], c["P"], c["h"], c["hk"], c["D"], c["sinks"], c["window"], c["ring"],
                          s.Q.to(DEV), s.K.to(DEV), s.V.to(DEV), O, Kcache=Kc, Vcache=Vc,
                          start=torch.tensor(s.start, **i32), counts=torch.tensor(s.counts, **i32),
                          workspace=space_for(c, flags) if space is None else space,
                          io_dtype=CODE[c["dtype"]], scale=scale, flags=flags)


def run(c, seed=0, scale=0.0, flags=0):
    print(f"[case] sink {c} scale {scale} flags {flags}", flush=True)
    s = Stream(c, seed)
    O = torch.full((c["B"], c["T"], c["P"], c["h"] * c["D"]), 777.0, dtype=TORCH[c["dtype"]], device=DEV)
    rows = O.clone()
    Kc, Vc = s.Kc.to(DEV), s.Vc.to(DEV)
    forward(s, c, O, Kc, Vc, scale, flags)
    torch.cuda.synchronize()
    ref, tol = s.reference(scale if scale > 0 else c["D"] ** -0.5)
    got = O.cpu().double()
    for b in range(c["B"]):
        n = s.counts[b]
        off = (got[b, :n] - ref[b, :n]).abs()
        assert (off <= tol[b, :n]).all(), f"stream {b}: {(off / (tol[b, :n] + 1e-300)).nan_to_num(1e9).max().item()} of the tolerance"
        assert same_bits(O[b, n:], rows[b, n:]), "rows behind the last new frame"
    Kw, Vw = s.caches()
    assert same_bits(Kc, Kw) and same_bits(Vc, Vw), "caches"
    return s, O


DIMS = [1, 5, 8, 16, 24, 32, 40, 48, 64, 72, 80, 96, 100, 104, 128, 136, 160, 176, 192, 200, 216, 232, 256, 264, 512]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", DIMS)
def test_one_frame_of_every_head_dim(D, dtype):
    run(case(dtype, T=1, P=5, h=3, D=D, sinks=2, window=9, start=40), D)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", DIMS)
def test_many_frames_of_every_head_dim(D, dtype):
    run(case(dtype, T=70, P=2, h=2, D=D, sinks=3, window=21, start=13), D)
    run(case(dtype, T=70, P=2, h=2, D=D, sinks=3, window=130, start=150), D)
    run(case(dtype, T=9, P=2, h=2, D=D, sinks=1, window=12, start=40), D)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 3, 4, 7, 8, 15, 16, 17, 31, 33, 64, 65, 130])
@pytest.mark.parametrize("sinks,window", [(0, 1), (0, 16), (1, 33), (4, 64), (17, 5), (5, 0), (0, 0), (40, 200)])
def test_windows_and_sinks(T, sinks, window, dtype):
    for start in (0, 3, 90):
        run(case(dtype, T=T, P=2, h=2, D=64, sinks=sinks, window=window, start=start), T + start)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("h,hk", [(1, 1), (2, 1), (6, 2), (8, 1), (12, 4), (16, 2), (20, 1), (5, 5)])
@pytest.mark.parametrize("T,window,start", [(1, 30, 100), (1, 700, 900), (3, 100, 50), (33, 40, 20), (100, 1000, 0)])
def test_shared_heads(T, window, start, h, hk, dtype):
    run(case(dtype, T=T, P=1, h=h, hk=hk, D=32, sinks=4, window=window, start=start), h + T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 64, 128])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_streams_of_different_lengths(T, D, dtype):
    starts, counts = [0, 1, 7, 300, 41, 1000], [T, max(0, T - 1), 0, T, 1, T // 2]
    run(case(dtype, B=6, T=T, P=3, h=4, hk=2, D=D, sinks=4, window=37, start=starts, counts=counts), T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,ring", [(1, 11), (5, 10), (5, 14), (5, 15), (40, 10), (40, 60), (25, 12)])
def test_rings_shorter_and_longer_than_a_call(T, ring, dtype):
    for start in (0, 2, 10, 11, 87):
        run(case(dtype, T=T, P=3, h=2, D=48, sinks=2, window=10, ring=ring, start=start), ring + start)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,P,h,hk,D,window,start", [(1, 1, 8, 2, 128, 5000, 6000), (1, 160, 8, 8, 160, 60, 77),
                                                     (2, 40, 8, 8, 80, 500, 600), (1, 700, 5, 5, 40, 16, 300),
                                                     (6, 1, 8, 1, 64, 3000, 2500), (300, 1, 4, 2, 128, 513, 100),
                                                     (48, 90, 5, 5, 64, 24, 0), (600, 1, 2, 1, 80, 2000, 0)])
def test_real_sizes(T, P, h, hk, D, window, start, dtype):
    run(case(dtype, B=2, T=T, P=P, h=h, hk=hk, D=D, sinks=4, window=window, start=start), T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 40])
def test_generic_kernel_and_scale(T, dtype):
    c = case(dtype, B=2, T=T, P=3, h=4, hk=2, D=64, sinks=2, window=30, start=[5, 64])
    run(c, 3, scale=0.4, flags=B.DSATTN_FLAG_FORCE_GENERIC)
    run(c, 3, scale=0.4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(2, 64), (40, 64), (70, 128), (40, 100)])
def test_what_a_query_does_not_see_does_not_reach_it(T, D, dtype):
    """Frames with infinities and NaN: the queries that see them are no numbers, all others as without."""
    c = case(dtype, T=T, P=2, h=2, D=D, sinks=2, window=7, start=20)
    clean, tol = Stream(c, 1).reference(D ** -0.5)
    hit = T // 2  # a new frame: queries hit .. hit + 6 see it
    for tensor, value in (("V", "nan"), ("V", "inf"), ("K", "nan"), ("K", "inf")):
        s = Stream(c, 1)
        getattr(s, tensor)[0, hit, 0, :] = float(value)      # position 0
        getattr(s, tensor + "c")[0, slot(17, 2, c["ring"]), 1, :] = float(value)  # an old frame, position 1: to frame 23
        O = torch.zeros(1, T, 2, 2 * D, dtype=TORCH[dtype], device=DEV)
        forward(s, c, O, s.Kc.to(DEV), s.Vc.to(DEV))
        torch.cuda.synchronize()
        bad = ~O.float().isfinite().cpu()
        want = torch.zeros(T, 2, dtype=torch.bool)
        want[hit:hit + 7, 0] = True
        want[:4, 1] = True
        if value == "nan" or tensor == "V":
            assert torch.equal(bad[0].all(-1), want) and torch.equal(bad[0].any(-1), want), (tensor, value)
        ok = ~want[None, :, :, None].expand_as(bad)
        assert ((O.cpu().double() - clean).abs() <= tol)[ok].all(), (tensor, value)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 40])
def test_large_scores(T, dtype):
    """Scores of some thousands: the running maximum has to hold them."""
    c = case(dtype, T=T, P=2, h=2, D=64, sinks=2, window=50, start=60)
    s = Stream(c, 2)
    s.Q, s.K, s.Kc = s.Q * 16, s.K * 16, s.Kc * 16
    O = torch.zeros(1, T, 2, 128, dtype=TORCH[dtype], device=DEV)
    forward(s, c, O, s.Kc.to(DEV), s.Vc.to(DEV))
    torch.cuda.synchronize()
    ref, tol = s.reference(64 ** -0.5)
    assert ((O.cpu().double() - ref).abs() <= tol + 1e-30).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_caches(dtype):
    c = case(dtype, B=2, T=45, P=3, h=2, D=64, sinks=3, window=12)
    s = Stream(c, 4)
    O = torch.zeros(2, 45, 3, 128, dtype=TORCH[dtype], device=DEV)
    B.dsattn_sink_forward(2, 45, 3, 2, 2, 64, 3, 12, None, s.Q.to(DEV), s.K.to(DEV), s.V.to(DEV), O,
                          workspace=space_for(c), io_dtype=CODE[dtype])
    torch.cuda.synchronize()
    ref, tol = s.reference(64 ** -0.5)
    assert ((O.cpu().double() - ref).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_frame_by_frame_is_the_whole_video(dtype):
    """One call over 60 frames, calls of 7 and calls of one, with a ring: the same video."""
    F, P, h, D, sinks, window = 60, 3, 2, 64, 3, 11
    whole = Stream(case(dtype, T=F, P=P, h=h, D=D, sinks=sinks, window=window), 6)
    ref, tol = whole.reference(D ** -0.5)
    for T in (60, 7, 1):
        c = case(dtype, T=T, P=P, h=h, D=D, sinks=sinks, window=window, ring=window + 3)
        Kc = torch.full((1, sinks + c["ring"], P, h * D), float("nan"), dtype=TORCH[dtype], device=DEV)
        Vc = Kc.clone()
        outs = []
        for f in range(0, F, T):
            part = Stream(c, 0)
            n = min(T, F - f)
            part.start, part.counts = [f], [n]
            for name in ("Q", "K", "V"):
                getattr(part, name)[:, :n] = getattr(whole, name)[:, f:f + n]
            O = torch.zeros(1, T, P, h * D, dtype=TORCH[dtype], device=DEV)
            forward(part, c, O, Kc, Vc)
            outs.append(O[:, :n])
        torch.cuda.synchronize()
        got = torch.cat(outs, 1).cpu().double()
        assert ((got - ref).abs() <= tol).all(), T


@pytest.mark.gpu
def test_starts_and_counts_outside_their_ranges_count_as_the_nearest():
    c = case("bf16", B=4, T=3, P=2, h=2, D=64, sinks=2, window=6, start=[0, 0, 0, 0], counts=[3, 0, 3, 3])
    s = Stream(c, 5)
    O, O2 = (torch.zeros(4, 3, 2, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    caches = [s.Kc.to(DEV), s.Vc.to(DEV), s.Kc.to(DEV), s.Vc.to(DEV)]
    forward(s, c, O, caches[0], caches[1])
    s.start, s.counts = [-5, -(1 << 31), 0, -1], [9, -2, (1 << 31) - 1, 3]
    forward(s, c, O2, caches[2], caches[3])
    torch.cuda.synchronize()
    assert same_bits(O, O2) and same_bits(caches[0], caches[2]) and same_bits(caches[1], caches[3])


@pytest.mark.gpu
@pytest.mark.parametrize("T,ring", [(1, 17), (3, 17), (40, 17), (40, 100), (90, 97)])
def test_the_largest_frame_numbers(T, ring):
    c = case("bf16", T=T, P=2, h=2, D=64, sinks=2, window=6, ring=ring)
    s, at = Stream(case("bf16", T=T, P=2, h=2, D=64, sinks=2, window=6, ring=ring, start=0x7fffffff - T - 1000), 5), 0x7fffffff - T
    s.start = [at]
    O = torch.zeros(1, T, 2, 128, dtype=torch.bfloat16, device=DEV)
    rng = torch.Generator().manual_seed(1)
    s.Kc, s.Vc = (torch.randn(s.Kc.shape, generator=rng).to(torch.bfloat16) for _ in range(2))
    Kc, Vc = s.Kc.to(DEV), s.Vc.to(DEV)
    forward(s, c, O, Kc, Vc)
    torch.cuda.synchronize()
    assert all(same_bits(got, want) for got, want in zip((Kc, Vc), s.caches()))
    frames = [0, 1] + list(range(at - 5, at + T))
    for t in range(T):
        a = at + t
        seen = [f for f in frames if f < 2 or a - 6 < f <= a]
        kv = [s.frame(0, f) for f in seen]
        k, v = (torch.stack([x[i] for x in kv]).double().reshape(-1, 2, 2, 64) for i in range(2))
        w = torch.softmax(torch.einsum("phd,jphd->phj", s.Q[0, t].double().reshape(2, 2, 64), k) / 8, -1)
        ref = torch.einsum("phj,jphd->phd", w, v).reshape(2, 128)
        assert ((O[0, t].cpu().double() - ref).abs() <= 0.03).all()  # (weights and output at 2^-8, |v| to 4.5)


def _desc(**kw):
    d = dict(streams=1, frames=2, spatial=3, heads=4, kv_heads=2, head_dim=32, sinks=1, window=4, ring=8,
             io_dtype=B.DSATTN_BF16, scale=0.0, flags=0)
    d.update(kw)
    return B.DsattnSinkDesc(**d)


BAD = [dict(streams=0), dict(frames=0), dict(spatial=0), dict(heads=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=513),
       dict(kv_heads=3), dict(kv_heads=8), dict(sinks=-1), dict(window=-1), dict(ring=3), dict(window=0, ring=0), dict(io_dtype=2),
       dict(scale=float("nan")), dict(scale=float("inf")), dict(flags=2), dict(heads=1 << 16, head_dim=32, kv_heads=1),
       dict(frames=(1 << 24) + 1), dict(ring=1 << 25), dict(streams=1 << 15), dict(spatial=1 << 30, ring=1 << 20)]


@pytest.mark.parametrize("kw", BAD)
def test_bad_descriptors_are_refused(kw):
    lib, n = B.load(), ctypes.c_size_t()
    assert lib.dsattn_sink_workspace(ctypes.byref(_desc(**kw)), ctypes.byref(n)) == B.DSATTN_EINVAL
    rc = lib.dsattn_sink_forward(ctypes.byref(_desc(**kw)), None, None, 0x10000, 0x20000, 0x30000, 0x40000, 0x50000,
                                 0x60000, 0x1000000, 1 << 40, None)
    assert rc == B.DSATTN_EINVAL and B.dsattn_last_error()


def test_bad_pointers_are_refused():
    lib = B.load()
    d = ctypes.byref(_desc())
    good = dict(start=0x100000, counts=0x110000, Q=0x120000, K=0x130000, V=0x140000, Kc=0x150000, Vc=0x160000, O=0x170000,
                ws=0x1000000, n=1 << 30)
    bad = [dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(Kc=None), dict(Vc=None), dict(Kc=None, Vc=None),
           dict(Q=0x120008), dict(K=0x130002), dict(V=0x140004), dict(O=0x170008), dict(Kc=0x150008), dict(Vc=0x160008),
           dict(ws=0x1000008), dict(start=0x100002), dict(counts=0x110001), dict(O=0x120010), dict(O=0x130000), dict(O=0x150000),
           dict(Kc=0x130010), dict(Vc=0x150010), dict(O=0x100000), dict(Kc=0x110000), dict(K=0x160010)]
    for kw in bad:
        a = {**good, **kw}
        rc = lib.dsattn_sink_forward(d, a["start"], a["counts"], a["Q"], a["K"], a["V"], a["Kc"], a["Vc"], a["O"], a["ws"],
                                     a["n"], None)
        assert rc == B.DSATTN_EINVAL, kw
    assert lib.dsattn_sink_workspace(d, None) == B.DSATTN_EINVAL


def test_a_short_workspace_is_refused():
    lib, need = B.load(), ctypes.c_size_t()
    for kw in (dict(frames=1, spatial=1, head_dim=128, window=16384, ring=16384), {}):
        d = _desc(**kw)
        assert lib.dsattn_sink_workspace(ctypes.byref(d), ctypes.byref(need)) == B.DSATTN_OK
        if need.value:
            for ws, n in ((1 << 45, need.value - 1), (None, need.value)):
                rc = lib.dsattn_sink_forward(ctypes.byref(d), 1 << 41, None, 1 << 42, 1 << 43, 1 << 44, 1 << 46, 1 << 47, 1 << 48,
                                             ws, n, None)
                assert rc == B.DSATTN_EINVAL and "workspace" in B.dsattn_last_error()


def test_binding_checks_tensors():
    t = dict(dtype=torch.bfloat16)
    q, k, cache = torch.zeros(1, 2, 3, 128, **t), torch.zeros(1, 2, 3, 64, **t), torch.zeros(1, 9, 3, 64, **t)
    i = torch.zeros(1, dtype=torch.int32)
    for kw in (dict(Q=k), dict(K=q), dict(V=k.float()), dict(O=q.float()), dict(Kcache=cache[:, :8]), dict(Vcache=cache.float()),
               dict(start=i.long()), dict(start=torch.zeros(2, dtype=torch.int32)), dict(counts=i.float()),
               dict(workspace=torch.zeros(4)), {}):
        a = {"Q": q, "K": k, "V": k, "O": q, "Kcache": cache, "Vcache": cache, "start": i, **kw}
        with pytest.raises(ValueError, match="dsattn_sink_forward"):
            B.dsattn_sink_forward(1, 2, 3, 4, 2, 32, 1, 4, 8, **a)


def test_the_definition_by_hand():
    """The visible frames of a small case, written out."""
    sees = {0: [0], 1: [0, 1], 4: [0, 1, 3, 4], 9: [0, 1, 8, 9]}  # two sinks, a window of two
    for a, frames in sees.items():
        assert [f for f in range(12) if 0 <= f <= a and (f < 2 or a - f < 2)] == frames
    assert [slot(f, 2, 3) for f in range(9)] == [0, 1, 2, 3, 4, 2, 3, 4, 2]
    assert np.array_equal([slot(f, 0, 4) for f in range(6)], [0, 1, 2, 3, 0, 1])
