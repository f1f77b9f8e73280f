"""Performance cases of the operators of a streaming transformer block over frames.

A case is a dict of plain values.  Its "op" says which entry point it goes through:

  rms   dsattn_rmsnorm: residual addition and root-mean-square norm, in 16, 32 or 8 bits
  lin   dsattn_linear_act: product with bias, activation, gate and residual
  sink  dsattn_sink_forward: causal attention over a window of frames and the first few, with its cache

listed() holds fixed cases, draw() gives more of the same ranges, prepare() makes inputs on the GPU from
a seed, run() makes one pass, work() counts what a pass cannot do without, and exact() computes the same
results in 64 bits.  Where `own` is false run() computes the operators with elementary torch operations
in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
E4M3_MAX = 448.0


def listed():
    return [
        # One frame of the U-Net's lowest level (5 x 8 positions of 1,280 channels): all latency.
        _rms("rms_frame_l4", rows=40, C=1280),
        # The headline tensor (2,304 frames x 10 x 16 positions), normalised into 8 bits for the next product.
        _rms("rms_2304f_l3_e4m3", rows=368640, C=1280, out="e4m3"),
        # The first layer of a timestep embedding: one row.
        _lin("lin_embedding", rows=1, c_in=320, c_out=1280, act="silu", residual=False),
        # One streamed frame of the headline level through an output projection with its residual.
        _lin("lin_frame_l3", rows=160, c_in=1280, c_out=1280, act="none"),
        # The gated feed-forward of 64 frames at the second level (20 x 32 positions, 640 channels).
        _lin("lin_64f_l2_gated", rows=40960, c_in=640, c_out=2560, act="gelu", gated=True, residual=False),
        # The way back from it, for clips of 24 frames of 9 x 15 positions: ragged in every tile.
        _lin("lin_192f_back", rows=25920, c_in=5120, c_out=1280, act="none"),
        # The gated feed-forward of 384 frames at the headline level, in 8 bits.
        _lin("lin_384f_l3_gated_e4m3", rows=61440, c_in=1280, c_out=5120, act="gelu", gated=True, residual=False,
             dtype="e4m3"),
        # fp32 tensors, 24 frames of 135 positions.
        _lin("lin_24f_f32", rows=3240, c_in=320, c_out=960, act="gelu_tanh", dtype="f32"),
        # One new frame at the headline level over its 4 first and 60 last frames.
        _sink("sink_frame_l3", T=1, P=160, heads=8, kv_heads=8, D=160, sinks=4, window=60, ring=64),
        # One new token of each of 16 streams over a long window: 32 heads on 8 of keys and values.
        _sink("sink_token_long", B=16, T=1, P=1, heads=32, kv_heads=8, D=128, sinks=4, window=16384, ring=16384),
        # A first chunk of 128 frames at the second level, nothing cached yet.
        _sink("sink_chunk_l2", T=128, P=640, heads=8, kv_heads=8, D=80, sinks=4, window=32, ring=40, first=True),
        # A long prompt of one position, window of 2,048.
        _sink("sink_prompt_long", B=2, T=8192, P=1, heads=16, kv_heads=4, D=128, sinks=4, window=2048, ring=2048,
              first=True),
    ]


def _rms(name=None, **kw):
    c = {"op": "rms", "dtype": "bf16", "out": "bf16", "residual": True, **kw}
    return {"name": name, **c} if name else c


def _lin(name=None, **kw):
    c = {"op": "lin", "dtype": "bf16", "gated": False, "bias": True, "residual": True, **kw}
    c.setdefault("out", "f32" if c["dtype"] == "f32" else "bf16")
    return {"name": name, **c} if name else c


def _sink(name=None, **kw):
    c = {"op": "sink", "dtype": "bf16", "B": 1, "first": False, "ragged": False, **kw}
    return {"name": name, **c} if name else c


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rms", "lin", "lin", "sink", "sink"])
    if op == "rms":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        C = rng.choice([rng.randrange(32, 192) * 8, _spread(rng, 40, 5120), 320, 640, 1280, 2560])
        rows = _spread(rng, 1, min(400000, 400_000_000 // C))
        return _rms(rows=rows, C=C, dtype=dtype, out=rng.choice([dtype, "e4m3"]), residual=rng.random() < 0.7)
    if op == "lin":
        dtype = rng.choice(["bf16", "bf16", "e4m3", "f32"])
        c_in = 16 * _spread(rng, 8, 320)
        c_out = 8 * _spread(rng, 8, 640)
        gated = rng.random() < 0.4
        most = (1 << 40) // (c_in * c_out * (2 if gated else 1)) // (16 if dtype == "f32" else 2)
        rows = _spread(rng, 1, max(1, min(65536, most)))
        return _lin(rows=rows, c_in=c_in, c_out=c_out, act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                    gated=gated, bias=rng.random() < 0.7, residual=rng.random() < 0.5, dtype=dtype)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kind = rng.choice(["frame", "frame", "chunk", "tokens", "prompt"])
    sinks = rng.choice([0, 1, 4, 4, rng.randrange(2, 17)])
    kv_heads = rng.choice([1, 2, 4, 8, 5])
    D = rng.choice([32, 40, 64, 80, 96, 128, 160])
    B = rng.choice([1, 1, 2, 3])
    if kind == "frame":  # a new frame, or a few, of many positions
        T, P, group = rng.choice([1, 1, 2, 4]), _spread(rng, 40, 1000), rng.choice([1, 1, 2])
        window = _spread(rng, 4, 160)
    elif kind == "chunk":  # a chunk of frames after others
        T, P, group = _spread(rng, 8, 160), _spread(rng, 16, 640), 1
        window = _spread(rng, 4, 160)
    elif kind == "tokens":  # one token, or some, of streams of one position
        T, P, group = rng.choice([1, 1, 1, rng.randrange(2, 9)]), 1, rng.choice([1, 2, 4, 8])
        window = _spread(rng, 64, 16384)
        B = rng.randrange(1, 17)
    else:
        T, P, group = _spread(rng, 256, 4096), 1, rng.choice([1, 2, 4])
        window = _spread(rng, 32, 4096)
        B = 1
    row = kv_heads * D * (4 if dtype == "f32" else 2)
    P = max(1, min(P, (1 << 30) // (4 * B * (T + sinks + window) * row)))
    return _sink(B=B, T=T, P=P, heads=kv_heads * group, kv_heads=kv_heads, D=D, sinks=sinks, window=window,
                 ring=window + T + rng.randrange(0, 9), dtype=dtype, first=rng.random() < 0.25,
                 ragged=rng.random() < 0.3)


# ------------------------------------------------------------------------------------- inputs

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _quantised(x):
    """Rows of x in 8 bits, and a scale for each."""
    scale = x.abs().amax(dim=-1, keepdim=True).clamp_min(1e-20) / E4M3_MAX
    return (x / scale).to(torch.float8_e4m3fn), scale.reshape(-1).contiguous()


def prepare(case, seed):
    g, c, op = _gen(seed), dict(case), case["op"]
    s = {"case": c}
    if op == "rms":
        t = _TORCH[c["dtype"]]
        rows, C = c["rows"], c["C"]
        # activations of a residual stream: rows of different size, some channels far larger than the rest
        size = torch.exp(0.5 * _randn(g, rows, 1))
        channel = torch.where(torch.rand(C, generator=g, device=DEV) < 0.01, 8.0, 1.0)
        s["X"] = (_randn(g, rows, C) * size * channel).to(t)
        s["R"] = _randn(g, rows, C).to(t) if c["residual"] else None
        s["gamma"] = 1.0 + 0.2 * _randn(g, C)
        s["total"] = torch.empty(rows, C, dtype=t, device=DEV) if c["residual"] else None
        s["Y"] = torch.empty(rows, C, dtype=_TORCH[c["out"]], device=DEV)
        s["scales"] = torch.empty(rows, device=DEV) if c["out"] == "e4m3" else None
    elif op == "lin":
        rows, c_in, c_out, sets = c["rows"], c["c_in"], c["c_out"], 2 if c["gated"] else 1
        x = _randn(g, rows, c_in)
        w = [_randn(g, c_out, c_in) * c_in ** -0.5 for _ in range(sets)]
        s["sx"] = s["sw"] = None
        if c["dtype"] == "e4m3":
            s["X"], s["sx"] = _quantised(x)
            pairs = [_quantised(a) for a in w]
            s["W"], s["sw"] = [a for a, _ in pairs], [b for _, b in pairs]
        else:
            s["X"], s["W"] = x.to(_TORCH[c["dtype"]]), [a.to(_TORCH[c["dtype"]]) for a in w]
        s["bias"] = [0.3 * _randn(g, c_out) for _ in range(sets)] if c["bias"] else None
        out = _TORCH[c["out"]]
        s["R"] = _randn(g, rows, c_out).to(out) if c["residual"] else None
        s["Y"] = torch.empty(rows, c_out, dtype=out, device=DEV)
    else:
        t = _TORCH[c["dtype"]]
        B, T, P, C, Ckv = c["B"], c["T"], c["P"], c["heads"] * c["D"], c["kv_heads"] * c["D"]
        slots = c["sinks"] + c["ring"]
        # projections of slowly varying latents: a part that all frames share, and one of their own
        s["Q"] = (_randn(g, 1, 1, P, C) + 0.5 * _randn(g, B, T, P, C)).to(t)
        base = _randn(g, 1, 1, P, Ckv)
        s["K"] = (base + 0.5 * _randn(g, B, T, P, Ckv)).to(t)
        s["V"] = _randn(g, B, T, P, Ckv).to(t)
        s["Kc"] = (base + 0.5 * _randn(g, B, slots, P, Ckv)).to(t)
        s["Vc"] = _randn(g, B, slots, P, Ckv).to(t)
        s["O"] = torch.zeros(B, T, P, C, dtype=t, device=DEV)
        lo, hi = (0, 1) if c["first"] else (c["sinks"] + c["window"] // 2, 3 * slots)
        s["start"] = torch.randint(lo, hi, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["counts"] = (torch.randint(1, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
                       if c["ragged"] else None)
    return s


def _code(B, name):
    return {"f32": B.DSATTN_F32, "bf16": B.DSATTN_BF16, "e4m3": B.DSATTN_E4M3}[name]


def _act_code(B, name):
    return {"none": B.DSATTN_ACT_NONE, "relu": B.DSATTN_ACT_RELU, "gelu": B.DSATTN_ACT_GELU,
            "gelu_tanh": B.DSATTN_ACT_GELU_TANH, "silu": B.DSATTN_ACT_SILU}[name]


def _sink_space(c):
    from paper_2406_16260_amd import binding as B
    return B.dsattn_sink_workspace(c["B"], c["T"], c["P"], c["heads"], c["kv_heads"], c["D"], c["sinks"],
                                   c["window"], c["ring"], io_dtype=_code(B, c["dtype"]))


# ------------------------------------------------------------------------------------- one pass

def run(s):
    return {"rms": _run_rms, "lin": _run_lin, "sink": _run_sink}[s["case"]["op"]](s)


def _run_rms(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        B.dsattn_rmsnorm(c["rows"], c["C"], s["X"], s["Y"], residual=s["R"], gamma=s["gamma"],
                         sum_out=s["total"], scales=s["scales"], io_dtype=_code(B, c["dtype"]), out_dtype=_code(B, c["out"]), eps=EPS)
        return {"sum": s["total"], "Y": s["Y"], "scales": s["scales"]}
    x = s["X"].float()
    if s["R"] is not None:
        x = x + s["R"].float()
    y = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * s["gamma"]
    total = x.to(s["X"].dtype) if s["R"] is not None else None
    if c["out"] != "e4m3":
        return {"sum": total, "Y": y.to(s["Y"].dtype), "scales": None}
    scale = (y.abs().amax(dim=-1, keepdim=True) / E4M3_MAX).clamp_min(2.0 ** -126)
    return {"sum": total, "Y": (y / scale).to(torch.float8_e4m3fn), "scales": scale.reshape(-1)}


def _run_lin(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        B.dsattn_linear_act(c["rows"], c["c_in"], c["c_out"], s["X"], s["W"], s["Y"], biases=s["bias"],
                            residual=s["R"], x_scales=s["sx"], w_scales=s["sw"], act=_act_code(B, c["act"]),
                            io_dtype=_code(B, c["dtype"]), out_dtype=_code(B, c["out"]))
        return s["Y"]
    y = _activated(_plain_product(s, 0), c["act"])
    if c["gated"]:
        y = y * _plain_product(s, 1)
    if s["R"] is not None:
        y = y + s["R"].float()
    return y.to(s["Y"].dtype)


def _plain_product(s, k):
    y = s["X"].float() @ s["W"][k].float().t()
    if s["sx"] is not None:
        y = y * s["sx"][:, None] * s["sw"][k]
    return y if s["bias"] is None else y + s["bias"][k]


def _activated(x, act):
    if act == "relu":
        return x.clamp_min(0)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _run_sink(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        if "space" not in s:  # a program allocates it once
            s["space"] = torch.empty(_sink_space(c), dtype=torch.uint8, device=DEV)
        B.dsattn_sink_forward(c["B"], c["T"], c["P"], c["heads"], c["kv_heads"], c["D"], c["sinks"], c["window"],
                              c["ring"], s["Q"], s["K"], s["V"], s["O"], Kcache=s["Kc"], Vcache=s["Vc"],
                              start=s["start"], counts=s["counts"], workspace=s["space"],
                              io_dtype=_code(B, c["dtype"]))
        return {"O": s["O"], "Kc": s["Kc"], "Vc": s["Vc"]}
    B, T, P, h, hk, D = (c[k] for k in ("B", "T", "P", "heads", "kv_heads", "D"))
    S, w, ring = c["sinks"], c["window"], c["ring"]
    start = s["start"].long()[:, None]
    counts = torch.full_like(start, T) if s["counts"] is None else s["counts"].long()[:, None]
    # the frames that any query sees: the first ones, and from the first query's window on
    sink = torch.arange(S, device=DEV).expand(B, S)
    near = start + torch.arange(1 - w, T, device=DEV)
    frame = torch.cat([sink, near], dim=1)
    there = torch.cat([sink < start + counts, (near >= S) & (near < start + counts)], dim=1)
    held = torch.where(frame < S, frame, S + (frame - S) % ring)
    at = torch.where(there, torch.where(frame < start, held, S + ring + frame - start), 0)
    rows = torch.arange(B, device=DEV)[:, None]
    k = torch.cat([s["Kc"], s["K"]], dim=1)[rows, at].float().reshape(B, -1, P, hk, D)
    v = torch.cat([s["Vc"], s["V"]], dim=1)[rows, at].float().reshape(B, -1, P, hk, D)
    q = s["Q"].float().reshape(B, T, P, hk, h // hk, D).permute(0, 2, 3, 4, 1, 5).reshape(B, P, hk, -1, D)
    score = torch.matmul(q, k.permute(0, 2, 3, 4, 1).contiguous()) * D ** -0.5
    score = score.reshape(B, P, hk, h // hk, T, -1)
    a, f = start[:, :, None] + torch.arange(T, device=DEV)[None, :, None], frame[:, None, :]
    seen = there[:, None, :] & (f <= a) & ((f < S) | (a - f < w))
    score = torch.where(seen[:, None, None, None], score, -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    e = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(dim=-1, keepdim=True)
    e = (e / torch.where(total == 0, 1.0, total)).reshape(B, P, hk, -1, frame.shape[1])
    o = torch.matmul(e, v.permute(0, 2, 3, 1, 4).contiguous())
    o = o.reshape(B, P, hk, h // hk, T, D).permute(0, 4, 1, 2, 3, 5).reshape(B, T, P, h * D)
    mine = torch.arange(T, device=DEV)[None, :] < counts
    o = torch.where(mine[:, :, None, None], o, 0.0).to(s["O"].dtype)
    # the last new frame of each slot goes into the cache
    new = start + torch.arange(T, device=DEV)
    slot = torch.where(new < S, new, S + (new - S) % ring)
    keep = mine & ((new < S) | (new + ring >= start + counts))
    b, t = torch.nonzero(keep, as_tuple=True)
    s["Kc"][b, slot[b, t]] = s["K"][b, t]
    s["Vc"][b, slot[b, t]] = s["V"][b, t]
    return {"O": o, "Kc": s["Kc"], "Vc": s["Vc"]}


# ------------------------------------------------------------------------------------- what a pass needs

_BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}


def work(case):
    c, op = case, case["op"]
    if op == "rms":
        n, es = c["rows"] * c["C"], _BYTES[c["dtype"]]
        moved = n * es * (3 if c["residual"] else 1) + n * _BYTES[c["out"]] + 4 * c["C"]
        return {"bytes": moved + (4 * c["rows"] if c["out"] == "e4m3" else 0), "flops": 4 * n}
    if op == "lin":
        sets, es, eo = 2 if c["gated"] else 1, _BYTES[c["dtype"]], _BYTES[c["out"]]
        rows, c_in, c_out = c["rows"], c["c_in"], c["c_out"]
        moved = (rows * c_in + sets * c_out * c_in) * es + rows * c_out * eo * (2 if c["residual"] else 1)
        if c["dtype"] == "e4m3":
            moved += 4 * (rows + sets * c_out)
        return {"bytes": moved + (4 * sets * c_out if c["bias"] else 0), "flops": 2 * rows * c_in * c_out * sets}
    # (streams that are past their window, or at their first frame; half of the new frames where they are ragged: the
    # starts and counts themselves are drawn by the seed)
    T, S, w, es = c["T"], c["sinks"], c["window"], _BYTES[c["dtype"]]
    T = (T + 1) // 2 if c["ragged"] else T
    n = c["B"] * c["P"]
    if c["first"]:
        seen = sum(min(t + 1, w + min(S, max(0, t + 1 - w))) for t in range(T))
        cached = 0
    else:
        seen, cached = T * (w + S), S + w - 1
    row, kv = c["heads"] * c["D"] * es, c["kv_heads"] * c["D"] * es
    return {"bytes": n * (2 * T * row + 2 * kv * (cached + 2 * min(T, S + c["ring"]))),
            "flops": 4 * n * c["heads"] * c["D"] * seen}


# ------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rms":
        v = s["X"].double() if s["R"] is None else s["X"].double() + s["R"].double()
        y = v / (v.pow(2).sum(-1, keepdim=True) / c["C"] + EPS).sqrt() * s["gamma"].double()
        out = {"sum": None if s["R"] is None else v, "Y": y, "scales": None}
        if c["out"] == "e4m3":
            scale = y.abs().max(-1).values / 448
            out.update(Y=y / scale[:, None], scales=scale)
        return out
    if c["op"] == "lin":
        parts = []
        for at in range(0, c["rows"], 8192):  # some rows at a time
            to = min(c["rows"], at + 8192)
            z = []
            for k, w in enumerate(s["W"]):
                w64 = w.double()
                if s["sw"] is not None:
                    w64 = w64 * s["sw"][k].double()[:, None]
                x64 = s["X"][at:to].double()
                if s["sx"] is not None:
                    x64 = x64 * s["sx"][at:to].double()[:, None]
                z.append(x64 @ w64.T + (0 if s["bias"] is None else s["bias"][k].double()))
            y = {"none": lambda v: v, "relu": lambda v: torch.maximum(v, torch.zeros_like(v)),
                 "gelu": lambda v: v * torch.special.ndtr(v),
                 "gelu_tanh": lambda v: v * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (v + 0.044715 * v ** 3)),
                 "silu": lambda v: v * torch.sigmoid(v)}[c["act"]](z[0])
            y = y * z[1] if c["gated"] else y
            parts.append(y if s["R"] is None else y + s["R"][at:to].double())
        return torch.cat(parts)
    B, T, P, h, hk, D = (c[k] for k in ("B", "T", "P", "heads", "kv_heads", "D"))
    S, w, ring = c["sinks"], c["window"], c["ring"]
    O = torch.zeros(B, T, P, h, D, dtype=torch.float64, device=DEV)
    starts = s["start"].tolist()
    counts = [T] * B if s["counts"] is None else s["counts"].tolist()

    def where(f):
        return f if f < S else S + (f - S) % ring

    for b in range(B):
        f0, n = starts[b], counts[b]
        for t0 in range(0, n, 512):  # some queries at a time, over the frames that the first and last of them see
            t1 = min(n, t0 + 512)
            first = max(0, f0 + t0 - w + 1)
            frames = list(range(min(S, first))) + list(range(first, f0 + t1))
            old = [where(f) for f in frames if f < f0]
            new = [f - f0 for f in frames if f >= f0]
            k, v = (torch.cat([cache[b, old], fresh[b, new]]).double().reshape(-1, P, hk, D)
                    for cache, fresh in ((s["Kc"], s["K"]), (s["Vc"], s["V"])))
            fr = torch.tensor(frames, device=DEV)
            aq = torch.arange(f0 + t0, f0 + t1, device=DEV)[:, None]
            hidden = (fr > aq) | ((fr >= S) & (fr <= aq - w))
            for g in range(hk):
                q = s["Q"][b, t0:t1].double().reshape(-1, P, hk, h // hk, D)[:, :, g].permute(1, 2, 0, 3)
                kk = k[:, :, g].permute(1, 2, 0).contiguous()[:, None]
                vv = v[:, :, g].permute(1, 0, 2).contiguous()[:, None]
                z = (torch.matmul(q, kk) / math.sqrt(D)).masked_fill(hidden, -math.inf)
                p = torch.softmax(z, dim=-1).nan_to_num(0.0)
                O[b, t0:t1].reshape(-1, P, hk, h // hk, D)[:, :, g] = torch.matmul(p, vv).permute(2, 0, 1, 3)
        for t in range(n):
            s["Kc"][b, where(f0 + t)] = s["K"][b, t]
            s["Vc"][b, where(f0 + t)] = s["V"][b, t]
    return {"O": O.reshape(B, T, P, h * D), "Kc": s["Kc"].double(), "Vc": s["Vc"].double()}
