"""Performance cases of the operators that train a recurrent streaming block: norm, recurrence over frames, products.

A case is a dict of plain values.  Its "op" says which entry point it goes through:

  ln        dsattn_layernorm: residual addition, layer norm with weight and bias
  ln_back   dsattn_layernorm_backward: gradients of the input, of weight and bias
  scan      dsattn_gated_scan: gated linear recurrence over frames, with the state it starts from and leaves
  scan_back dsattn_gated_scan_backward: gradients of inputs, gate logits and starting state
  lin_back  dsattn_linear_act_backward: gradients of a (gated) product with bias and activation, from its inputs

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
STEP = 16  # frames between the states that the recurrence keeps for its backward pass


def listed():
    return [
        # One frame of the U-Net's lowest level (5 x 8 positions of 1,280 channels): all latency.
        _ln("ln_frame_l4", rows=40, C=1280),
        # The headline tensor, 2,304 frames x 10 x 16 positions, with the residual's addition.
        _ln("ln_2304f_l3", rows=368640, C=1280),
        # Training on 64 frames at the second level (20 x 32 positions, 640 channels): the norm's way back.
        _ln("ln_64f_l2_back", back=True, rows=40960, C=640),
        # The same in fp32 for 24 frames of 9 x 15 positions.
        _ln("ln_24f_f32_back", back=True, rows=3240, C=320, dtype="f32"),
        # One new frame at the headline level: the state of every position and channel moves on by a step.
        _scan("scan_frame_l3", T=1, P=160, C=1280),
        # A chunk of 384 frames at the second level.
        _scan("scan_384f_l2", T=384, P=640, C=640, mode="mean"),
        # Two long sequences of one position: few channels for the many steps.
        _scan("scan_long", B=2, T=16384, P=1, C=1280, mode="norm"),
        # Training on 384 frames of 10 x 16 positions.
        _scan("scan_384f_l3_back", back=True, T=384, P=160, C=1280, mode="mean"),
        # Sequences of different lengths in one batch, fp32.
        _scan("scan_ragged_f32_back", back=True, B=4, T=4095, P=1, C=640, dtype="f32", ragged=True, mode="norm"),
        # One frame through a product with SiLU.
        _lin("lin_frame_l3_back", rows=160, c_in=1280, c_out=1280, act="silu"),
        # The gated feed-forward of 64 frames at the second level.
        _lin("lin_64f_l2_gated_back", rows=40960, c_in=640, c_out=2560, act="gelu", gated=True),
        # The product that follows it, for clips of 24 frames of 9 x 15 positions: ragged in every tile.
        _lin("lin_192f_back", rows=25920, c_in=5120, c_out=1280, act="none"),
    ]


def _named(name, c):
    return {"name": name, **c} if name else c


def _ln(name=None, back=False, **kw):
    return _named(name, {"op": "ln_back" if back else "ln", "dtype": "bf16", "residual": True, **kw})


def _scan(name=None, back=False, **kw):
    return _named(name, {"op": "scan_back" if back else "scan", "dtype": "bf16", "B": 1, "mode": "mean", "ragged": False, **kw})


def _lin(name=None, **kw):
    return _named(name, {"op": "lin_back", "dtype": "bf16", "gated": False, "bias": True, **kw})


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["ln", "ln", "scan", "scan", "lin", "lin"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    back = rng.random() < 0.5
    if op == "ln":
        C = rng.choice([rng.randrange(32, 192) * 8, _spread(rng, 40, 5120), 320, 640, 1280, 2560])
        rows = _spread(rng, 1, min(200000, 200_000_000 // C))
        return _ln(back=back, rows=rows, C=C, dtype=dtype, residual=rng.random() < 0.7)
    if op == "scan":
        mode, ragged = rng.choice(["sum", "mean", "norm"]), rng.random() < 0.3
        C = rng.choice([8 * _spread(rng, 5, 160), _spread(rng, 40, 1280), 320, 640, 1280])
        if rng.random() < 0.5:  # frames of many positions
            B, T, P = rng.choice([1, 1, 2]), _spread(rng, 1, 384), _spread(rng, 16, 640)
        else:                   # sequences of one
            B, T, P = rng.randrange(1, 9), _spread(rng, 1, 16384), 1
        T = max(1, min(T, 40_000_000 // (B * P * C)))
        return _scan(back=back, B=B, T=T, P=P, C=C, dtype=dtype, mode=mode, ragged=ragged)
    c_in, c_out, gated = 8 * _spread(rng, 8, 640), 8 * _spread(rng, 8, 640), rng.random() < 0.5
    most = (1 << 37) // (c_in * c_out * (2 if gated else 1)) // (16 if dtype == "f32" else 1)
    rows = _spread(rng, 1, max(1, min(65536, most)))
    return _lin(rows=rows, c_in=c_in, c_out=c_out, act=rng.choice(["none", "gelu", "gelu_tanh", "silu"]), gated=gated,
                bias=rng.random() < 0.7, dtype=dtype)


# ------------------------------------------------------------------------------------- inputs

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    c, op, t = dict(case), case["op"], _TORCH[case["dtype"]]
    s = {"case": c}
    if op in ("ln", "ln_back"):
        rows, C = c["rows"], c["C"]
        # activations of a residual stream: rows of different size and mean, some channels far larger than the rest
        size = torch.exp(0.5 * randn(rows, 1))
        channel = torch.where(torch.rand(C, generator=g, device=DEV) < 0.01, 8.0, 1.0)
        s["X"] = ((randn(rows, C) * channel + 0.5 * randn(rows, 1)) * size).to(t)
        s["R"] = randn(rows, C).to(t) if c["residual"] else None
        s["gamma"], s["beta"] = 1.0 + 0.2 * randn(C), 0.2 * randn(C)
        if op == "ln":
            s["total"] = torch.empty_like(s["X"]) if c["residual"] else None
            s["Y"] = torch.empty_like(s["X"])
        else:
            s["dY"] = randn(rows, C).to(t)
            s["dsum"] = randn(rows, C).to(t) if c["residual"] else None
            s["dX"] = torch.empty_like(s["X"])
            s["dgamma"], s["dbeta"] = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    elif op in ("scan", "scan_back"):
        B, T, P, C = c["B"], c["T"], c["P"], c["C"]
        # gates that remember over some frames to some hundreds, another span for every channel
        span = 6.0 * torch.rand(C, generator=g, device=DEV) - 0.5
        s["X"] = randn(B, T, P, C).to(t)
        s["G"] = (span + randn(B, T, P, C)).to(t)
        s["h0"] = randn(B, P, C)
        s["counts"] = (torch.randint(1, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
                       if c["ragged"] else None)
        if op == "scan":
            s["Y"], s["hT"] = torch.zeros_like(s["X"]), torch.empty_like(s["h0"])
        else:
            s["dY"], s["dhT"] = randn(B, T, P, C).to(t), randn(B, P, C)
            s["dX"], s["dG"], s["dh0"] = torch.zeros_like(s["X"]), torch.zeros_like(s["X"]), torch.empty_like(s["h0"])
            s["states"] = _states(s)  # the forward pass leaves them
    else:
        rows, c_in, c_out, sets = c["rows"], c["c_in"], c["c_out"], 2 if c["gated"] else 1
        s["X"] = randn(rows, c_in).to(t)
        s["W"] = [(randn(c_out, c_in) * c_in ** -0.5).to(t) for _ in range(sets)]
        s["bias"] = [0.3 * randn(c_out) for _ in range(sets)] if c["bias"] else None
        s["dY"] = randn(rows, c_out).to(t)
        s["dX"] = torch.empty_like(s["X"])
        s["dW"] = [torch.empty_like(m) for m in s["W"]]
        s["db"] = [torch.empty(c_out, device=DEV) for _ in range(sets)] if c["bias"] else None
    return s


def _code(B, name):
    return {"f32": B.DSATTN_F32, "bf16": B.DSATTN_BF16}[name]


def _mode_code(B, name):
    return {"sum": B.DSATTN_SCAN_SUM, "mean": B.DSATTN_SCAN_MEAN, "norm": B.DSATTN_SCAN_NORM}[name]


def _act_code(B, name):
    return {"none": B.DSATTN_ACT_NONE, "gelu": B.DSATTN_ACT_GELU, "gelu_tanh": B.DSATTN_ACT_GELU_TANH,
            "silu": B.DSATTN_ACT_SILU}[name]


def _states(s):
    """The state in front of every STEP frames, in 32 bits."""
    T = s["X"].shape[1]
    h = _all_states(s)
    return torch.cat([s["h0"][:, None], h[:, STEP - 1:T - 1:STEP]], dim=1).contiguous()


def _space(s, size):
    if "space" not in s:  # a program allocates it once
        s["space"] = torch.empty(size(), dtype=torch.uint8, device=DEV)
    return s["space"]


# ------------------------------------------------------------------------------------- one pass

def run(s):
    return {"ln": _run_ln, "ln_back": _run_ln_back, "scan": _run_scan, "scan_back": _run_scan_back,
            "lin_back": _run_lin_back}[s["case"]["op"]](s)


def _centred(s):
    x = s["X"].float()
    if s["R"] is not None:
        x = x + s["R"].float()
    d = x - x.mean(dim=-1, keepdim=True)
    return x, d, torch.rsqrt((d * d).mean(dim=-1, keepdim=True) + EPS)


def _run_ln(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        B.dsattn_layernorm(c["rows"], c["C"], s["X"], s["Y"], residual=s["R"], gamma=s["gamma"], beta=s["beta"],
                           sum_out=s["total"], io_dtype=_code(B, c["dtype"]), eps=EPS)
        return {"sum": s["total"], "Y": s["Y"]}
    x, d, rstd = _centred(s)
    return {"sum": x.to(s["X"].dtype) if s["R"] is not None else None,
            "Y": (d * rstd * s["gamma"] + s["beta"]).to(s["X"].dtype)}


def _run_ln_back(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        code = _code(B, c["dtype"])
        space = _space(s, lambda: B.dsattn_layernorm_backward_workspace(c["rows"], c["C"], io_dtype=code))
        B.dsattn_layernorm_backward(c["rows"], c["C"], s["X"], s["dY"], s["dX"], residual=s["R"], gamma=s["gamma"],
                                    dsum=s["dsum"], dgamma=s["dgamma"], dbeta=s["dbeta"], workspace=space,
                                    io_dtype=code, eps=EPS)
        return {"dX": s["dX"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    _, d, rstd = _centred(s)
    xhat, dy = d * rstd, s["dY"].float()
    dxhat = dy * s["gamma"]
    dx = rstd * (dxhat - dxhat.mean(dim=-1, keepdim=True) - xhat * (dxhat * xhat).mean(dim=-1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dX": dx.to(s["X"].dtype), "dgamma": (dy * xhat).sum(dim=0), "dbeta": dy.sum(dim=0)}


def _gates(s):
    """What is kept of the state, what is let in, and the second's derivative by the gate's logit."""
    g, mode = s["G"].float(), s["case"]["mode"]
    keep, leave = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    if mode == "mean":
        return keep, leave, -keep * leave
    if mode == "norm":
        return keep, torch.sqrt(leave * (1 + keep)), -keep * keep * torch.sqrt(leave / (1 + keep))
    return keep, torch.ones_like(keep), torch.zeros_like(keep)


def _scanned(a, b):
    """h_t = a_t h_(t-1) + b_t along dimension 1, from 0 on: spans of 1, 2, 4, .. steps joined."""
    span = 1
    while span < a.shape[1]:
        b = torch.cat([b[:, :span], b[:, span:] + a[:, span:] * b[:, :-span]], dim=1)
        a = torch.cat([a[:, :span], a[:, span:] * a[:, :-span]], dim=1)
        span *= 2
    return b


def _mine(s):
    """Which frames of each stream there are: [B, T, 1, 1]."""
    B, T = s["X"].shape[:2]
    if s["counts"] is None:
        return torch.ones(B, T, 1, 1, dtype=torch.bool, device=DEV)
    return (torch.arange(T, device=DEV) < s["counts"][:, None])[:, :, None, None]


def _all_states(s):
    keep, let, _ = _gates(s)
    mine = _mine(s)
    keep, b = torch.where(mine, keep, 1.0), torch.where(mine, let * s["X"].float(), 0.0)
    b[:, 0] = b[:, 0] + keep[:, 0] * s["h0"]
    return _scanned(keep, b)


def _run_scan(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        code, shape = _code(B, c["dtype"]), (c["B"], c["T"], c["P"], c["C"])
        space = _space(s, lambda: B.dsattn_gated_scan_workspace(*shape, io_dtype=code))
        B.dsattn_gated_scan(*shape, s["X"], s["G"], s["Y"], mode=_mode_code(B, c["mode"]), start_state=s["h0"],
                            end_state=s["hT"], counts=s["counts"], workspace=space, io_dtype=code)
        return {"Y": s["Y"], "hT": s["hT"]}
    h = _all_states(s)  # (behind a stream's end the state stays)
    return {"Y": torch.where(_mine(s), h, 0.0).to(s["X"].dtype), "hT": h[:, -1].contiguous()}


def _run_scan_back(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        code, shape = _code(B, c["dtype"]), (c["B"], c["T"], c["P"], c["C"])
        space = _space(s, lambda: B.dsattn_gated_scan_workspace(*shape, io_dtype=code))
        B.dsattn_gated_scan_backward(*shape, s["X"], s["G"], s["states"], s["dY"], s["dX"], s["dG"],
                                     mode=_mode_code(B, c["mode"]), dend_state=s["dhT"], dstart_state=s["dh0"],
                                     counts=s["counts"], workspace=space, io_dtype=code)
        return {"dX": s["dX"], "dG": s["dG"], "dh0": s["dh0"]}
    keep, let, dlet = _gates(s)
    mine, x = _mine(s), s["X"].float()
    h = _all_states(s)
    before = torch.cat([s["h0"][:, None], h[:, :-1]], dim=1)
    # D_t = dY_t + a_(t+1) D_(t+1), from the last frame on
    a = torch.where(mine, keep, 1.0).flip(1)
    late = torch.cat([torch.ones_like(a[:, :1]), a[:, :-1]], dim=1)
    d = torch.where(mine, s["dY"].float(), 0.0).flip(1)
    d[:, 0] = d[:, 0] + s["dhT"]
    d = _scanned(late, d).flip(1)
    dkeep = keep * (1 / (1 + torch.exp(s["G"].float())))
    dx = torch.where(mine, d * let, 0.0)
    dg = torch.where(mine, d * (before * dkeep + x * dlet), 0.0)
    first = torch.where(mine[:, 0], keep[:, 0], 1.0)
    return {"dX": dx.to(s["X"].dtype), "dG": dg.to(s["X"].dtype), "dh0": d[:, 0] * first}


def _run_lin_back(s):
    c = s["case"]
    if own:
        from paper_2406_16260_amd import binding as B
        code, act = _code(B, c["dtype"]), _act_code(B, c["act"])
        space = _space(s, lambda: B.dsattn_linear_act_backward_workspace(c["rows"], c["c_in"], c["c_out"], n_w=len(s["W"]),
                                                                         act=act, io_dtype=code))
        B.dsattn_linear_act_backward(c["rows"], c["c_in"], c["c_out"], s["X"], s["W"], s["dY"], dX=s["dX"], dWs=s["dW"],
                                     dbiases=s["db"], biases=s["bias"], act=act, workspace=space, io_dtype=code)
        return {"dX": s["dX"], "dW": s["dW"], "db": s["db"]}
    x, w, dy = s["X"].float(), [m.float() for m in s["W"]], s["dY"].float()
    z = [x @ m.t() + (0.0 if s["bias"] is None else s["bias"][k]) for k, m in enumerate(w)]
    y, slope = _activated(z[0], c["act"])
    dz = [dy * z[1] * slope, dy * y] if c["gated"] else [dy * slope]
    dx = dz[0] @ w[0]
    for k in range(1, len(w)):
        dx = dx + dz[k] @ w[k]
    return {"dX": dx.to(s["X"].dtype), "dW": [(d.t() @ x).to(s["X"].dtype) for d in dz],
            "db": None if s["bias"] is None else [d.sum(dim=0) for d in dz]}


def _activated(x, act):
    """The activation and its derivative."""
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
        return x * p, p + x * torch.exp(-0.5 * x * x) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (x + 0.044715 * x * x * x))
        return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 0.134145 * x * x)
    if act == "silu":
        p = 1 / (1 + torch.exp(-x))
        return x * p, p * (1 + x * (1 - p))
    return x, torch.ones_like(x)


# ------------------------------------------------------------------------------------- what a pass needs

_BYTES = {"f32": 4, "bf16": 2}


def work(case):
    c, op, es = case, case["op"], _BYTES[case["dtype"]]
    if op in ("ln", "ln_back"):
        n = c["rows"] * c["C"]
        tensors = (4 if c["residual"] else 2) if op == "ln" else (5 if c["residual"] else 3)
        return {"bytes": n * es * tensors + (8 if op == "ln" else 12) * c["C"], "flops": (8 if op == "ln" else 16) * n}
    if op in ("scan", "scan_back"):
        # (half of the frames where the streams are ragged: their counts are drawn by the seed)
        T = (c["T"] + 1) // 2 if c["ragged"] else c["T"]
        n, state = c["B"] * T * c["P"] * c["C"], c["B"] * c["P"] * c["C"]
        if op == "scan":
            return {"bytes": n * es * 3 + 8 * state, "flops": 8 * n}
        return {"bytes": n * es * 5 + 4 * state * (2 + (T + STEP - 1) // STEP), "flops": 20 * n}
    sets, rows, c_in, c_out = 2 if c["gated"] else 1, c["rows"], c["c_in"], c["c_out"]
    moved = (2 * rows * c_in + rows * c_out + 2 * sets * c_out * c_in) * es
    # the product itself again (but where its derivative is 1), and the two of its gradient
    products = 2 if c["act"] == "none" and not c["gated"] else 3
    return {"bytes": moved + (8 * sets * c_out if c["bias"] else 0), "flops": 2 * rows * c_in * c_out * sets * products}


# ------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    c, op, s = case, case["op"], prepare(case, seed)
    if op in ("ln", "ln_back"):
        v = s["X"].double() if s["R"] is None else s["X"].double() + s["R"].double()
        var, mu = torch.var_mean(v, dim=-1, correction=0, keepdim=True)
        n = (v - mu) / (var + EPS).sqrt()
        if op == "ln":
            return {"sum": None if s["R"] is None else v, "Y": torch.addcmul(s["beta"].double(), n, s["gamma"].double())}
        dy = s["dY"].double()
        e = dy * s["gamma"].double()
        # the part of e across 1 and n
        e = e - e.sum(-1, keepdim=True) / c["C"]
        e = e - n * ((e * n).sum(-1, keepdim=True) / c["C"])
        dx = e / (var + EPS).sqrt()
        return {"dX": dx if s["dsum"] is None else dx + s["dsum"].double(), "dgamma": (dy * n).sum(0),
                "dbeta": dy.sum(0)}
    if op in ("scan", "scan_back"):
        return _exact_scan(c, s)
    x = s["X"].double().requires_grad_()
    w = [m.double().requires_grad_() for m in s["W"]]
    b = None if s["bias"] is None else [m.double().requires_grad_() for m in s["bias"]]
    act = {"none": lambda v: v, "gelu": lambda v: v * torch.special.ndtr(v),
           "gelu_tanh": lambda v: v * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (v + 0.044715 * v ** 3)),
           "silu": lambda v: v * torch.sigmoid(v)}[c["act"]]
    for at in range(0, c["rows"], 8192):  # some rows at a time
        to = min(c["rows"], at + 8192)
        z = [torch.nn.functional.linear(x[at:to], m, None if b is None else b[k]) for k, m in enumerate(w)]
        y = act(z[0]) * z[1] if c["gated"] else act(z[0])
        y.backward(s["dY"][at:to].double())
    return {"dX": x.grad, "dW": [m.grad for m in w], "db": None if b is None else [m.grad for m in b]}


def _exact_scan(c, s):
    T = c["T"]
    counts = [T] * c["B"] if s["counts"] is None else s["counts"].tolist()
    h = s["h0"].double()
    out, before = torch.zeros(s["X"].shape, dtype=torch.float64, device=DEV), []

    def gate(t, on):
        a = torch.sigmoid(s["G"][on, t].double())
        ia = torch.sigmoid(-s["G"][on, t].double())
        w = {"sum": torch.ones_like(a), "mean": ia, "norm": torch.sqrt(ia * (1 + a))}[c["mode"]]
        dw = {"sum": torch.zeros_like(a), "mean": -a * ia, "norm": -a * a * ia / torch.sqrt(ia * (1 + a))}[c["mode"]]
        return a, ia, w, dw

    ragged = s["counts"] is not None
    for t in range(T):  # one frame after the other
        on = [b for b in range(c["B"]) if t < counts[b]] if ragged else slice(None)
        if ragged and not on:
            break
        a, _, w, _ = gate(t, on)
        if c["op"] == "scan_back":
            before.append(h[on])
        nxt = a * h[on] + w * s["X"][on, t].double()
        h = h.clone() if ragged else h
        if ragged:
            h[on] = nxt
        else:
            h = nxt
        out[on, t] = nxt
    if c["op"] == "scan":
        return {"Y": out, "hT": h}
    dx, dg, d = torch.zeros_like(out), out, s["dhT"].double()
    dg.zero_()
    for t in reversed(range(len(before))):
        on = [b for b in range(c["B"]) if t < counts[b]] if ragged else slice(None)
        a, ia, w, dw = gate(t, on)
        now = d[on] + s["dY"][on, t].double()
        dx[on, t] = now * w
        dg[on, t] = now * (before[t] * a * ia + dw * s["X"][on, t].double())
        d = d.clone()
        d[on] = now * a
    return {"dX": dx, "dG": dg, "dh0": d}
