"""The projections and rotary positions around the attention layer: what is measured of them.

A video transformer's attention layer is a matrix product into queries, keys and values, their RMS
norm and rotation by the token's (time, height, width) position, the attention itself, and a matrix
product back whose result is scaled by a gate and added to the residual stream. A case is one call of
`linear` (y = residual + gate * act(x w^T + bias)), of `rotary` (norm and rotation of queries and
keys), or of the backward pass of either.

Sizes are those of the layer of 40 heads of 128 (5,120 features) over 21 x 45 x 80 tokens that this
repository is built for, what one of eight GPUs holds of its sequence (9,450 tokens), its text tokens
(256), single rows as a time embedding has, and small, odd and ragged ones in both types.
"""
import math

import torch

own = False

GPU = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _linear(name, what, dtype, batch, n, k, o, act="none", bias=True, gate="none", residual=False, pre=False):
    c = {"what": what, "dtype": dtype, "batch": batch, "n": n, "k": k, "o": o, "act": act, "bias": bias, "gate": gate,
         "residual": residual, "pre": pre}
    return {"name": name, **c} if name else c


def _rotary(name, what, dtype, batch, heads, d, t, h, w, tail, sections, norm, halves=False, listed_positions=False,
            first=0, count=0):
    c = {"what": what, "dtype": dtype, "batch": batch, "heads": heads, "d": d, "t": t, "h": h, "w": w, "tail": tail,
         "st": sections[0], "sh": sections[1], "sw": sections[2], "norm": norm, "halves": halves,
         "positions": listed_positions, "first": first, "count": count or t * h * w}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the first product of a time embedding: one row, SiLU; launch latency
        _linear("linear_one_row", "linear", "bf16", 1, 1, 256, 5120, act="silu"),
        # the modulation of a layer, six vectors for a guided pair: every weight read for two rows
        _linear("linear_modulation", "linear", "bf16", 2, 1, 5120, 30720),
        # text tokens into the model's width
        _linear("linear_text", "linear", "bf16", 1, 256, 4096, 5120, act="gelu_tanh"),
        # queries, keys and values of the whole sequence in one product: the largest call
        _linear("linear_qkv", "linear", "bf16", 1, 75600, 5120, 15360),
        # the projection out of the layer on one of eight GPUs: gate and residual, two clips at once
        _linear("linear_out_gated", "linear", "bf16", 2, 9450, 5120, 5120, gate="batch", residual=True),
        # fp32, no size a multiple of anything, everything in the epilogue
        _linear("linear_f32_odd", "linear", "f32", 3, 701, 1003, 1541, act="gelu", gate="token", residual=True, pre=True),
        # a step of training of the layer's way in to the wide product of its feed-forward part
        _linear("linear_backward_wide", "linear_backward", "bf16", 1, 9450, 5120, 20480, act="gelu_tanh"),
        # fp32 gradients of a small gated product, ragged rows
        _linear("linear_backward_f32", "linear_backward", "f32", 2, 777, 640, 1000, act="silu", gate="batch"),
        # queries and keys of the whole sequence out of the fused projection, norm across the heads
        _rotary("rotary_layer", "rotary", "bf16", 1, 40, 128, 21, 45, 80, 0, (22, 21, 21), "token"),
        # one new token of each of eight clips, positions from a list
        _rotary("rotary_one_token", "rotary", "bf16", 8, 40, 128, 1, 1, 1, 0, (22, 21, 21), "token", listed_positions=True),
        # fp32 heads of 64 with text tokens, halves paired, norm of each head; a ragged share of the sequence
        _rotary("rotary_f32_tail", "rotary", "f32", 2, 5, 64, 9, 31, 45, 77, (8, 12, 11), "head", halves=True, first=1234, count=4321),
        # the gradient of one of eight GPUs' share
        _rotary("rotary_backward_shard", "rotary_backward", "bf16", 1, 40, 128, 21, 45, 80, 0, (22, 21, 21), "token", first=9450, count=9450),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    what = rng.choice(["linear", "linear", "linear", "linear_backward", "linear_backward", "rotary", "rotary", "rotary_backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    batch = rng.choice([1, 1, 2, 3])
    if what.startswith("linear"):
        step = rng.choice([64, 8, 1])
        k = max(step, log(48, 20480) // step * step)
        o = max(step, log(48, 20480) // step * step)
        most = min((4e12 if dtype == "bf16" else 2e11) / (2.0 * k * o * batch), 5e8 / ((k + 4 * o) * batch))
        n = log(1, max(2, min(75600 // batch, int(most))))
        if rng.random() < 0.25:
            n = rng.randint(1, 40)
        act = rng.choice(["none", "silu", "gelu", "gelu_tanh"])
        gate = rng.choice(["none", "batch", "token"])
        return _linear("", what, dtype, batch, n, k, o, act=act, bias=rng.random() < 0.8, gate=gate,
                       residual=what == "linear" and rng.random() < 0.5, pre=what == "linear" and rng.random() < 0.3)
    d = rng.choice([128, 128, 64])
    heads = rng.choice([1, 2, 5, 8, 12, 24, 40, 40])
    n = log(1, max(2, min(75600, int(75600 * 40 * 128 / (2 * heads * d * batch)))))
    tail = rng.choice([0, 0, rng.randint(1, 256)])
    t = rng.randint(1, 21)
    w = max(1, int(math.sqrt(n / t * 16 / 9)))
    h = max(1, n // (t * w))
    whole = t * h * w
    first = rng.choice([0, rng.randint(0, whole - 1)])
    count = whole - first if rng.random() < 0.5 else rng.randint(1, whole - first)
    half = d // 2
    st = rng.randint(0, half // 3)
    sh = rng.randint(1, half // 3)
    sw = rng.choice([half - st - sh, rng.randint(0, half - st - sh)])
    return _rotary("", what, dtype, batch, heads, d, t, h, w, tail, (st, sh, sw), rng.choice(["none", "head", "token"]),
                   halves=rng.random() < 0.4, listed_positions=rng.random() < 0.3, first=first, count=count)


# ------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=GPU)
    g.manual_seed(int(seed))
    return g


def _grid_positions(c):
    i = torch.arange(c["first"], c["first"] + c["count"], device=GPU)
    return torch.stack([i // (c["h"] * c["w"]), i // c["w"] % c["h"], i % c["w"]], 1)


def _frequencies(c):
    """One frequency for each pair of each axis: 10000^(-i / pairs of the axis)."""
    return torch.cat([10000.0 ** (-torch.arange(s, dtype=torch.float64, device=GPU) / max(s, 1)) for s in (c["st"], c["sh"], c["sw"])])


def prepare(case, seed):
    c, dt, g = case, DT[case["dtype"]], _generator(seed)

    def normal(*shape, scale=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device=GPU) * scale + mean).to(dt)

    s = {"case": c}
    if c["what"].startswith("linear"):
        B, n, k, o = c["batch"], c["n"], c["k"], c["o"]
        s["x"] = normal(B, n, k)
        s["w"] = normal(o, k, scale=k ** -0.5)
        s["bias"] = normal(o, scale=0.1) if c["bias"] else None
        s["gate"] = None if c["gate"] == "none" else normal(B, o, scale=0.5) if c["gate"] == "batch" else normal(B, n, o, scale=0.5)
        s["residual"] = normal(B, n, o) if c["residual"] else None
        if c["what"] == "linear_backward":
            s["dy"] = normal(B, n, o)
            z = s["x"].float().reshape(B * n, k) @ s["w"].float().t()
            s["pre"] = (z if s["bias"] is None else z + s["bias"].float()).reshape(B, n, o).to(dt)
        return s
    B, H, d, n = c["batch"], c["heads"], c["d"], c["count"] + c["tail"]
    # the fused projection's output: a token's queries of all heads, its keys, its values
    s["qkv"] = normal(B, n, 3, H, d, scale=1.5)
    s["q"], s["k"] = s["qkv"][:, :, 0].transpose(1, 2), s["qkv"][:, :, 1].transpose(1, 2)
    size = {"none": 0, "head": d, "token": H * d}[c["norm"]]
    s["weights"] = [normal(size, scale=0.2, mean=1.0) for _ in range(2)] if size else None
    s["inv_freq"] = _frequencies(c)
    if c["positions"]:
        # positions of tokens that lie anywhere in a long generation, each clip's own
        far = torch.tensor([4000, 90, 160], device=GPU)
        s["positions"] = (torch.rand(B, c["count"], 3, generator=g, device=GPU) * far).floor().int()
    if c["what"] == "rotary_backward":
        s["grads"] = [normal(B, H, n, d) for _ in range(2)]
    return s


# ------------------------------------------------------------------------------------ plain forms
def _act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    if act == "gelu_tanh":
        c = (2.0 / math.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _linear_plain(s):
    c, dt = s["case"], DT[s["case"]["dtype"]]
    B, n, k, o = c["batch"], c["n"], c["k"], c["o"]
    z = (s["x"].float().reshape(B * n, k) @ s["w"].float().t()).reshape(B, n, o)
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["gate"] is not None:
        y = y * (s["gate"].float() if c["gate"] == "token" else s["gate"].float()[:, None])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(dt), "pre": z.to(dt)} if c["pre"] else {"y": y.to(dt)}


def _linear_backward_plain(s):
    c, dt = s["case"], DT[s["case"]["dtype"]]
    B, n, k, o = c["batch"], c["n"], c["k"], c["o"]
    dy, z = s["dy"].float(), s["pre"].float()
    dz = dy * _act_slope(z, c["act"])
    r = {}
    if s["gate"] is not None:
        da = dy * _act(z, c["act"])
        dz = dz * (s["gate"].float() if c["gate"] == "token" else s["gate"].float()[:, None])
        r["dgate"] = (da if c["gate"] == "token" else da.sum(1)).to(dt)
    dz = dz.reshape(B * n, o)
    if s["bias"] is not None:
        r["dbias"] = dz.sum(0).to(dt)
    r["dx"] = (dz @ s["w"].float()).reshape(B, n, k).to(dt)
    r["dw"] = (dz.t() @ s["x"].float().reshape(B * n, k)).to(dt)
    return r


def _angles(s):
    """cos and sin [batch or 1, rotated tokens, pairs] in 32 bits, of angles in 64."""
    c = s["case"]
    pos = s["positions"].double() if c["positions"] else _grid_positions(c).double()[None]
    axis = torch.repeat_interleave(torch.arange(3, device=GPU), torch.tensor([c["st"], c["sh"], c["sw"]], device=GPU))
    a = pos[:, :, axis] * s["inv_freq"]
    return a.cos().float(), a.sin().float()


def _rotate(x, cos, sin, halves):
    """x [B, H, tokens, d] with the first pairs rotated: (2p, 2p + 1), or (p, p + pairs)."""
    P = cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    y = x.clone()
    a, b = (x[..., :P], x[..., P:2 * P]) if halves else (x[..., 0:2 * P:2], x[..., 1:2 * P:2])
    u, v = a * cos - b * sin, a * sin + b * cos
    if halves:
        y[..., :P], y[..., P:2 * P] = u, v
    else:
        y[..., 0:2 * P:2], y[..., 1:2 * P:2] = u, v
    return y


def _norm_weight(s, i):
    c = s["case"]
    w = s["weights"][i].float()
    return w if c["norm"] == "head" else w.reshape(c["heads"], 1, c["d"])


EPS = 1e-6


def _norm_factor(x, norm):
    over = (3,) if norm == "head" else (1, 3)
    return torch.rsqrt((x * x).mean(over, keepdim=True) + EPS)


def _rotary_plain(s):
    c, dt = s["case"], DT[s["case"]["dtype"]]
    cos, sin = _angles(s)
    out = []
    for i, x in enumerate((s["q"], s["k"])):
        x = x.float()
        if c["norm"] != "none":
            x = x * _norm_factor(x, c["norm"]) * _norm_weight(s, i)
        m = c["count"]
        out.append(torch.cat([_rotate(x[:, :, :m], cos, sin, c["halves"]), x[:, :, m:]], 2).to(dt))
    return {"q": out[0], "k": out[1]}


def _rotary_backward_plain(s):
    c, dt = s["case"], DT[s["case"]["dtype"]]
    cos, sin = _angles(s)
    r = {"dx": [], "dweight": []}
    for i, (x, dy) in enumerate(zip((s["q"], s["k"]), s["grads"])):
        dy, m = dy.float(), c["count"]
        du = torch.cat([_rotate(dy[:, :, :m], cos, -sin, c["halves"]), dy[:, :, m:]], 2)
        if c["norm"] == "none":
            r["dx"].append(du.to(dt))
            continue
        over = (3,) if c["norm"] == "head" else (1, 3)
        x = x.float()
        f = _norm_factor(x, c["norm"])
        xh, dxh = x * f, du * _norm_weight(s, i)
        r["dx"].append((f * (dxh - xh * (dxh * xh).mean(over, keepdim=True))).to(dt))
        dw = (du * xh).sum(2).sum(0)  # [heads, d]
        r["dweight"].append((dw.sum(0) if c["norm"] == "head" else dw.reshape(-1)).to(dt))
    return r


# ------------------------------------------------------------------------------------ one pass
def _rotary_arguments(s):
    c = s["case"]
    kw = {"n_tail": c["tail"], "norm": None if c["norm"] == "none" else c["norm"], "weights": s["weights"], "eps": EPS,
          "halves": c["halves"]}
    if c["positions"]:
        kw["positions"] = s["positions"]
    else:
        kw["grid"], kw["first"] = (c["t"], c["h"], c["w"]), c["first"]
    return (s["inv_freq"], (c["st"], c["sh"], c["sw"])), kw


def run(s):
    c = s["case"]
    if not own:
        return {"linear": _linear_plain, "linear_backward": _linear_backward_plain, "rotary": _rotary_plain,
                "rotary_backward": _rotary_backward_plain}[c["what"]](s)
    import paper_2603_08982_amd as sv

    if c["what"] == "linear":
        y, pre = sv.linear(s["x"], s["w"], s["bias"], act=c["act"], gate=s["gate"], residual=s["residual"], want_pre=c["pre"])
        return {"y": y, "pre": pre} if c["pre"] else {"y": y}
    if c["what"] == "linear_backward":
        want = ["dx", "dw"] + (["dbias"] if s["bias"] is not None else []) + (["dgate"] if s["gate"] is not None else [])
        return sv.linear_backward(s["dy"], s["x"], s["w"], pre=s["pre"], act=c["act"], gate=s["gate"], want=want)
    args, kw = _rotary_arguments(s)
    if c["what"] == "rotary":
        q, k = sv.rotary([s["q"], s["k"]], *args, **kw)
        return {"q": q, "k": k}
    dx, dweight = sv.rotary_backward(s["grads"], [s["q"], s["k"]], *args, **kw)
    return {"dx": dx, "dweight": dweight if c["norm"] != "none" else []}


def work(case):
    c, e = case, 4 if case["dtype"] == "f32" else 2
    if c["what"].startswith("linear"):
        m = c["batch"] * c["n"]
        rows = m * c["o"]  # values of an output-shaped tensor
        gate = {"none": 0, "batch": c["batch"] * c["o"], "token": rows}[c["gate"]]
        vectors = (c["o"] if c["bias"] else 0) + gate
        if c["what"] == "linear":
            moved = m * c["k"] + c["o"] * c["k"] + vectors + rows * (1 + c["residual"] + c["pre"])
            return {"bytes": e * moved, "flops": 2.0 * m * c["o"] * c["k"]}
        needs_pre = c["act"] != "none" or c["gate"] != "none"
        moved = 2 * (m * c["k"] + c["o"] * c["k"] + vectors) + rows * (1 + needs_pre)
        return {"bytes": e * moved, "flops": 4.0 * m * c["o"] * c["k"]}
    values = 2 * c["batch"] * c["heads"] * (c["count"] + c["tail"]) * c["d"]
    back = c["what"] == "rotary_backward"
    positions = 12 * c["batch"] * c["count"] if c["positions"] else 0
    return {"bytes": e * values * (2 + (back and c["norm"] != "none")) + positions, "flops": (12.0 if back else 8.0) * values}


# ------------------------------------------------------------------------------------ 64 bits
def _exact_linear(s, c):
    x, w = s["x"].double().flatten(0, 1), s["w"].double()
    phi = {"none": lambda z: z, "silu": lambda z: z * torch.sigmoid(z), "gelu": lambda z: z * 0.5 * torch.erfc(-z / math.sqrt(2.0)),
           "gelu_tanh": lambda z: z * torch.sigmoid(math.sqrt(8.0 / math.pi) * (z + 0.044715 * z ** 3))}[c["act"]]
    z = torch.mm(x, w.t()).unflatten(0, (c["batch"], c["n"]))
    if s["bias"] is not None:
        z += s["bias"].double()
    y = phi(z)
    if c["gate"] == "batch":
        y = y * s["gate"].double().unsqueeze(1)
    elif c["gate"] == "token":
        y = y * s["gate"].double()
    if c["residual"]:
        y = y + s["residual"].double()
    return {"y": y, "pre": z} if c["pre"] else {"y": y}


def _exact_linear_backward(s, c):
    z, dy = s["pre"].double(), s["dy"].double()
    if c["act"] == "none":
        a, slope = z, torch.ones_like(z)
    elif c["act"] == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        a, slope = z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:  # z sigmoid(u(z)): slope sigmoid(u) + z sigmoid'(u) u'
        c0 = math.sqrt(8.0 / math.pi)
        u, du = (z, 1.0) if c["act"] == "silu" else (c0 * (z + 0.044715 * z ** 3), c0 * (1 + 0.134145 * z ** 2))
        sg = torch.sigmoid(u)
        a, slope = z * sg, sg + z * sg * torch.sigmoid(-u) * du
    r = {}
    dz = slope * dy
    if c["gate"] == "batch":
        dz = dz * s["gate"].double().unsqueeze(1)
        r["dgate"] = torch.einsum("bno,bno->bo", dy, a)
    elif c["gate"] == "token":
        dz = dz * s["gate"].double()
        r["dgate"] = dy * a
    dz = dz.flatten(0, 1)
    if s["bias"] is not None:
        r["dbias"] = dz.sum(0)
    r["dx"] = torch.mm(dz, s["w"].double()).unflatten(0, (c["batch"], c["n"]))
    r["dw"] = torch.mm(s["x"].double().flatten(0, 1).t(), dz).t()
    return r


def _exact_turn(s, c, x, sign):
    """Pairs as complex numbers times e^(sign i angle); what is not rotated stays."""
    m, P = c["count"], c["st"] + c["sh"] + c["sw"]
    if c["positions"]:
        pos = s["positions"].double()
    else:
        i = torch.arange(c["count"], device=GPU) + c["first"]
        hw = c["h"] * c["w"]
        pos = torch.stack([i.div(hw, rounding_mode="floor"), (i % hw).div(c["w"], rounding_mode="floor"), i % c["w"]], -1).double()[None]
    f = s["inv_freq"].split([c["st"], c["sh"], c["sw"]])
    angle = torch.cat([pos[..., k:k + 1] * f[k] for k in range(3)], -1)[:, None]
    turn = torch.polar(torch.ones_like(angle), sign * angle)
    y = x.clone()
    v = x[:, :, :m, :2 * P]
    if c["halves"]:
        t = torch.complex(v[..., :P].contiguous(), v[..., P:].contiguous()) * turn
        y[:, :, :m, :2 * P] = torch.cat([t.real, t.imag], -1)
    else:
        t = torch.view_as_complex(v.reshape(*v.shape[:-1], P, 2).contiguous()) * turn
        y[:, :, :m, :2 * P] = torch.view_as_real(t).flatten(-2)
    return y


def _exact_scale(x, c):
    if c["norm"] == "head":
        return (x.square().sum(-1, keepdim=True) / c["d"] + EPS) ** -0.5
    return (x.square().sum(-1, keepdim=True).sum(1, keepdim=True) / (c["d"] * c["heads"]) + EPS) ** -0.5


def _exact_weight(s, c, i):
    w = s["weights"][i].double()
    return w.view(1, 1, 1, -1) if c["norm"] == "head" else w.view(1, c["heads"], 1, c["d"])


def _exact_rotary(s, c):
    r = {}
    for i, name in enumerate("qk"):
        x = s[name].double()
        if c["norm"] != "none":
            x = x * _exact_scale(x, c) * _exact_weight(s, c, i)
        r[name] = _exact_turn(s, c, x, 1.0)
    return r


def _exact_rotary_backward(s, c):
    r = {"dx": [], "dweight": []}
    for i, name in enumerate("qk"):
        du = _exact_turn(s, c, s["grads"][i].double(), -1.0)
        if c["norm"] == "none":
            r["dx"].append(du)
            continue
        x = s[name].double()
        f = _exact_scale(x, c)
        g = du * _exact_weight(s, c, i)
        dot = (g * x).sum(-1, keepdim=True)
        count = c["d"]
        if c["norm"] == "token":
            dot, count = dot.sum(1, keepdim=True), c["d"] * c["heads"]
        r["dx"].append(f * g - f ** 3 * x * dot / count)
        per = (du * x * f).sum((0, 2))
        r["dweight"].append(per.sum(0) if c["norm"] == "head" else per.flatten())
    return r


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "linear_backward": _exact_linear_backward, "rotary": _exact_rotary,
            "rotary_backward": _exact_rotary_backward}[case["what"]](s, case)
