"""The layer norm around the attention layer and dense attention with masks: what is measured of them.

A video transformer's layer begins with a layer norm that the time embedding modulates, attends to the text tokens of its
prompt, whose number differs from prompt to prompt, and is trained on clips packed one behind the other in one sequence;
generated frame by frame, its tokens see the text and what came before them. A case is one call of `layer_norm`, of
`attention`, or of the backward pass of either.

Sizes are those of the layer of 40 heads of 128 (5,120 features) over 75,600 tokens that this repository is built for, what
one of eight GPUs holds of its sequence (9,450 tokens), padded texts, single tokens over a long past, and small, odd and
ragged ones in both types. Documents (packed clips, padded texts) are cut at places that a number in the case fixes.
"""
import math
import random

import torch

own = False

GPU = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _norm(name, what, dtype, batch, n, c, affine, mod):
    """mod: "none", "batch" (one scale and shift for a clip) or "token"."""
    r = {"what": what, "dtype": dtype, "batch": batch, "n": n, "c": c, "affine": affine, "mod": mod}
    return {"name": name, **r} if name else r


def _attn(name, what, dtype, batch, heads, kv, d, nq, nk, docs=0, cut=0, causal=False, prefix=0, cap=0.0, slopes=False, lse=False):
    """docs: documents of a batch entry (0: all rows are one); cut: places of their ends; prefix: the longest prefix."""
    r = {"what": what, "dtype": dtype, "batch": batch, "heads": heads, "kv": kv, "d": d, "nq": nq, "nk": nk, "docs": docs,
         "cut": cut, "causal": causal, "prefix": prefix, "cap": cap, "slopes": slopes, "lse": lse}
    return {"name": name, **r} if name else r


def listed():
    return [
        # a single token of a guided pair: launch latency
        _norm("norm_one_token", "layer_norm", "bf16", 2, 1, 5120, False, "batch"),
        # the whole sequence in front of the attention layer, modulated by the time embedding: the largest norm
        _norm("norm_modulated", "layer_norm", "bf16", 1, 75600, 5120, False, "batch"),
        # fp32, odd rows, weight and bias, each token with a time of its own
        _norm("norm_f32_odd", "layer_norm", "f32", 3, 701, 1003, True, "token"),
        # a step of training on one of eight GPUs, all gradients
        _norm("norm_backward_shard", "layer_norm_backward", "bf16", 1, 9450, 5120, True, "batch"),
        # fp32 gradients of the norm in front of the cross attention, ragged rows
        _norm("norm_backward_f32", "layer_norm_backward", "f32", 2, 777, 1541, True, "none"),
        # cross attention of a guided pair to its padded texts
        _attn("attn_text", "attention", "bf16", 2, 40, 40, 128, 37800, 512, docs=1, cut=3),
        # clips of several lengths packed into one sequence, with padding behind them
        _attn("attn_packed", "attention", "bf16", 1, 40, 40, 128, 9450, 9450, docs=4, cut=11, lse=True),
        # generation in order: text as prefix, capped scores, shared key and value heads
        _attn("attn_prefix", "attention", "bf16", 1, 40, 8, 128, 8704, 8704, docs=1, cut=7, causal=True, prefix=256, cap=50.0),
        # the next token of each of eight clips over a long past, distance bias: serving
        _attn("attn_one_token", "attention", "bf16", 8, 40, 8, 128, 1, 32760, docs=1, cut=5, causal=True, slopes=True),
        # fp32, small heads, nothing a multiple of anything
        _attn("attn_f32_odd", "attention", "f32", 2, 6, 2, 64, 1237, 1237, docs=3, cut=2, slopes=True, lse=True),
        # a step of training on packed clips: the largest gradients
        _attn("attn_backward_packed", "attention_backward", "bf16", 1, 16, 16, 128, 9450, 9450, docs=4, cut=11),
        # fp32 gradients with everything in the scores, shared heads
        _attn("attn_backward_f32", "attention_backward", "f32", 1, 8, 4, 64, 1531, 1531, docs=2, cut=9, causal=True, prefix=77, cap=30.0,
              slopes=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    what = rng.choice(["layer_norm", "layer_norm_backward", "attention", "attention", "attention", "attention_backward", "attention_backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    batch = rng.choice([1, 1, 2, 3])
    if what.startswith("layer_norm"):
        step = rng.choice([64, 8, 1])
        c = max(step, log(48, 20480) // step * step)
        mod = rng.choice(["none", "batch", "batch", "token"])
        most = 75600 * 5120 // (batch * c * (2 if dtype == "f32" else 1) * (2 if what.endswith("backward") else 1) * (3 if mod == "token" else 1))
        return _norm("", what, dtype, batch, log(1, max(2, min(200000, most))), c, rng.random() < 0.5, mod)
    kv = rng.choice([1, 2, 4, 8, 12])
    heads = kv * rng.choice([1, 1, 2, 3, 5, 8])
    d = rng.choice([128, 128, 64])
    back = what.endswith("backward")
    pairs = (9e8 if back else 2.2e9) * (0.1 if dtype == "f32" else 1) / (batch * heads)
    rows = (1.5e8 if back else 3e8) * (0.5 if dtype == "f32" else 1) / (batch * d)  # of all heads
    least = 32 if back else 1  # gradients through a softmax of one key are differences of equal numbers
    kind = rng.choice(["self", "self", "self", "cross", "few"])
    if kind == "self":
        nq = nk = log(least, max(2 * least, int(min(math.sqrt(pairs), rows / heads))))
    elif kind == "cross":
        nk = log(least, 1024)
        nq = log(1, max(2, int(min(75600, pairs / nk, rows / heads))))
    else:
        nq = rng.randint(1, 40)
        nk = max(nq, log(32, int(max(64, min(131072, pairs / nq, rows / kv)))))
    docs = rng.choice([0, 1, rng.randint(2, 9) if nk > 9 * least else 1]) if kind == "self" else rng.choice([0, 1])
    causal = kind != "cross" and rng.random() < 0.5
    prefix = rng.choice([0, rng.randint(1, 256)]) if causal else 0
    return _attn("", what, dtype, batch, heads, kv, d, nq, nk, docs=docs, cut=rng.randint(0, 10**6), causal=causal, prefix=prefix,
                 cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=kind != "cross" and rng.random() < 0.4, lse=not back and rng.random() < 0.4)


# ------------------------------------------------------------------------------------ inputs
def _documents(c):
    """Ends of the documents of each batch entry, (queries', keys'), each docs + 1 numbers, and the documents' prefixes."""
    rng = random.Random(c["cut"])
    q, k, p = [], [], []
    for _ in range(c["batch"]):
        if c["docs"] == 0:
            q.append([0, c["nq"]])
            k.append([0, c["nk"]])
        elif c["docs"] == 1:  # padded keys; where queries and keys are the same tokens the queries too
            n = max(1, int(c["nk"] * rng.uniform(0.5, 1.0)))
            k.append([0, n])
            q.append([0, n if c["nq"] == c["nk"] else c["nq"]])
        else:  # packed, up to a twentieth of padding behind the last
            n = max(1, int(c["nk"] * rng.uniform(0.95, 1.0)))
            ends = [0] + sorted(rng.randint(0, n) for _ in range(c["docs"] - 1)) + [n]
            q.append(ends)
            k.append(ends)
        p.append([rng.randint(0, c["prefix"]) for _ in range(max(1, c["docs"]))])
    return q, k, p


def _pairs(c):
    """Pairs of a query and a key that it sees, of one head of the whole batch, and the keys and queries in documents."""
    q, k, p = _documents(c)
    pairs = 0
    for qe, ke, pe in zip(q, k, p):
        for t in range(len(pe)):
            nq, nk = qe[t + 1] - qe[t], ke[t + 1] - ke[t]
            if not c["causal"]:
                pairs += nq * nk
            else:
                seen = torch.arange(nq) + nk - nq + 1
                pairs += int(seen.clamp(min=min(nk, pe[t])).clamp(min=0, max=nk).sum())
    return pairs, sum(e[-1] for e in k), sum(e[-1] for e in q)


def prepare(case, seed):
    c, dt = case, DT[case["dtype"]]
    g = torch.Generator(device=GPU)
    g.manual_seed(int(seed))

    def normal(*shape, scale=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device=GPU) * scale + mean).to(dt)

    s = {"case": c}
    if c["what"].startswith("layer_norm"):
        B, n, w = c["batch"], c["n"], c["c"]
        # a residual stream: channels of different means and widths
        s["x"] = (torch.randn(B, n, w, generator=g, device=GPU) * (0.5 + 2.0 * torch.rand(w, generator=g, device=GPU))
                  + torch.randn(w, generator=g, device=GPU)).to(dt)
        s["weight"], s["bias"] = (normal(w, scale=0.2, mean=1.0), normal(w, scale=0.1)) if c["affine"] else (None, None)
        shape = {"none": None, "batch": (B, w), "token": (B, n, w)}[c["mod"]]
        s["scale"], s["shift"] = (normal(*shape, scale=0.3), normal(*shape, scale=0.3)) if shape else (None, None)
        if c["what"] == "layer_norm_backward":
            s["dy"] = normal(B, n, w)
        return s
    B, H, Hk, d, nq, nk = c["batch"], c["heads"], c["kv"], c["d"], c["nq"], c["nk"]
    if nq == nk:  # the fused projection's output: a token's queries of all heads, its keys, its values
        q, k, v = normal(B, nq, H + 2 * Hk, d).split([H, Hk, Hk], 2)
    else:
        q = normal(B, nq, H, d)
        k, v = normal(B, nk, 2 * Hk, d).split([Hk, Hk], 2)
    s["q"], s["k"], s["v"] = (t.transpose(1, 2) for t in (q, k, v))
    qe, ke, p = (torch.tensor(e, dtype=torch.int32, device=GPU) for e in _documents(c))
    s["q_offsets"], s["k_offsets"] = (qe, ke) if c["docs"] else (None, None)
    s["prefix"] = p if c["prefix"] else None
    # slopes from 2^-1 or less downwards, a factor from head to head
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H + 1, device=GPU) / H) if c["slopes"] else None
    if c["what"] == "attention_backward":
        s["o"], s["lse"] = _attention_plain(s)
        s["dy"] = normal(B, H, nq, d)
    return s


# ------------------------------------------------------------------------------------ plain forms
def _over_tokens(s, name):
    """scale or shift, for every token."""
    t = s[name].float()
    return t if s["case"]["mod"] == "token" else t[:, None]


def _normalised(s):
    x = s["x"].float()
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _layer_norm_plain(s):
    u, _ = _normalised(s)
    if s["weight"] is not None:
        u = u * s["weight"].float() + s["bias"].float()
    if s["scale"] is not None:
        u = u * (1.0 + _over_tokens(s, "scale")) + _over_tokens(s, "shift")
    return {"y": u.to(s["x"].dtype)}


def _layer_norm_backward_plain(s):
    c, dt = s["case"], s["x"].dtype
    h, r = _normalised(s)
    dy = s["dy"].float()
    out, du = {}, dy
    if s["scale"] is not None:
        u = h * s["weight"].float() + s["bias"].float() if c["affine"] else h
        dscale = dy * u
        out["dscale"] = (dscale if c["mod"] == "token" else dscale.sum(1)).to(dt)
        out["dshift"] = (dy if c["mod"] == "token" else dy.sum(1)).to(dt)
        du = dy * (1.0 + _over_tokens(s, "scale"))
    g = du
    if c["affine"]:
        out["dweight"], out["dbias"] = (du * h).sum((0, 1)).to(dt), du.sum((0, 1)).to(dt)
        g = du * s["weight"].float()
    out["dx"] = (r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))).to(dt)
    return out


def _ranges(s):
    """For every query the keys that it sees, [lo, hi), and its position among the keys; each [B,1,Nq,1]."""
    c = s["case"]
    i = torch.arange(c["nq"], device=GPU)[None]
    if c["docs"]:
        qe, ke = s["q_offsets"].long(), s["k_offsets"].long()
    else:
        qe, ke = (torch.tensor([[0, n]], device=GPU).expand(c["batch"], 2) for n in (c["nq"], c["nk"]))
    # the query's document: the last that begins at or before it and is not over
    t = ((i[:, :, None] >= qe[:, None, 1:]).sum(-1)).clamp(max=qe.shape[1] - 2)
    i = i.expand(t.shape[0], -1)
    q0, q1, lo, hi = qe.gather(1, t), qe.gather(1, t + 1), ke.gather(1, t), ke.gather(1, t + 1)
    at = i - q0 + (hi - lo) - (q1 - q0) + lo
    if c["causal"]:
        seen = at + 1
        if s["prefix"] is not None:
            seen = torch.maximum(seen, lo + s["prefix"].long().gather(1, t))
        hi = torch.minimum(hi, seen)
    hi = torch.where((i >= q0) & (i < q1), hi, lo)
    return tuple(r[:, None, :, None] for r in (lo, hi, at))


def _group(t, kv):
    """[B,H,N,..] as [B,kv,H/kv*N,..]: the rows of the query heads that share a key head."""
    return t.reshape(t.shape[0], kv, -1, *t.shape[3:])


def _scores(s):
    """Scores [B,H,Nq,Nk] with -inf where nothing is seen, and the slope of the cap (None without one)."""
    c = s["case"]
    z = torch.matmul(_group(s["q"].float(), c["kv"]), s["k"].float().transpose(2, 3)) * c["d"] ** -0.5
    z = z.reshape(c["batch"], c["heads"], c["nq"], c["nk"])
    slope = None
    if c["cap"]:
        th = torch.tanh(z / c["cap"])
        z = c["cap"] * th
        slope = 1.0 - th * th if c["what"] == "attention_backward" else None
    lo, hi, at = _ranges(s)
    j = torch.arange(c["nk"], device=GPU)
    if c["slopes"]:
        z = z - s["slopes"][:, None, None] * (at - j).abs().float()
    return z.masked_fill((j < lo) | (j >= hi), -math.inf), slope


def _attention_plain(s):
    c = s["case"]
    z, _ = _scores(s)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(z - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(_group(p, c["kv"]), s["v"].float()).reshape(s["q"].shape)
    return torch.where(l > 0, o / l, 0.0).to(s["q"].dtype), (m + torch.log(l))[..., 0]


def _attention_backward_plain(s):
    c, dt, kv = s["case"], s["q"].dtype, s["case"]["kv"]
    z, slope = _scores(s)
    lse = s["lse"][..., None]
    p = torch.exp(z - torch.where(lse == -math.inf, 0.0, lse))
    dy = s["dy"].float()
    ds = torch.matmul(_group(dy, kv), s["v"].float().transpose(2, 3)).reshape(z.shape)
    ds = p * (ds - (dy * s["o"].float()).sum(-1, keepdim=True))
    if slope is not None:
        ds = ds * slope
    ds, p = _group(ds * c["d"] ** -0.5, kv), _group(p, kv)
    dq = torch.matmul(ds, s["k"].float()).reshape(s["q"].shape)
    dk = torch.matmul(ds.transpose(2, 3), _group(s["q"].float(), kv))
    dv = torch.matmul(p.transpose(2, 3), _group(dy, kv))
    return {"dq": dq.to(dt), "dk": dk.to(dt), "dv": dv.to(dt)}


# ------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if not own:
        if c["what"] == "attention":
            o, lse = _attention_plain(s)
            return {"o": o, "lse": lse} if c["lse"] else {"o": o}
        return {"layer_norm": _layer_norm_plain, "layer_norm_backward": _layer_norm_backward_plain,
                "attention_backward": _attention_backward_plain}[c["what"]](s)
    import paper_2603_08982_amd as sv

    if c["what"] == "layer_norm":
        return {"y": sv.layer_norm(s["x"], s["weight"], s["bias"], scale=s["scale"], shift=s["shift"], eps=EPS)}
    if c["what"] == "layer_norm_backward":
        want = ["dx"] + (["dweight", "dbias"] if c["affine"] else []) + (["dscale", "dshift"] if c["mod"] != "none" else [])
        return sv.layer_norm_backward(s["dy"], s["x"], s["weight"], s["bias"], scale=s["scale"], eps=EPS, want=want)
    kw = {"cap": c["cap"] or None, "slopes": s["slopes"], "causal": c["causal"], "prefix": s["prefix"],
          "q_offsets": s["q_offsets"], "k_offsets": s["k_offsets"]}
    if c["what"] == "attention":
        o, lse = sv.attention(s["q"], s["k"], s["v"], want_lse=c["lse"], **kw)
        return {"o": o, "lse": lse} if c["lse"] else {"o": o}
    return sv.attention_backward(s["dy"], s["q"], s["k"], s["v"], s["o"], s["lse"], **kw)


def work(case):
    c, e = case, 4 if case["dtype"] == "f32" else 2
    back = c["what"].endswith("backward")
    if c["what"].startswith("layer_norm"):
        rows = c["batch"] * c["n"]
        vectors = 2 * c["c"] * c["affine"] + 2 * c["c"] * {"none": 0, "batch": c["batch"], "token": rows}[c["mod"]]
        if back and c["mod"] == "token":  # the shift is not read, its gradient is written
            vectors += c["c"] * rows
        elif back:
            vectors *= 2
        return {"bytes": e * (rows * c["c"] * (3 if back else 2) + vectors), "flops": (15.0 if back else 8.0) * rows * c["c"]}
    pairs, keys, queries = _pairs(c)
    tensors = c["d"] * (c["heads"] * queries, c["kv"] * keys)[0], c["d"] * c["kv"] * keys
    moved = e * (4 * tensors[0] + 4 * tensors[1] if back else 2 * tensors[0] + 2 * tensors[1])
    moved += 4 * c["heads"] * queries * (1 if back or c["lse"] else 0)
    return {"bytes": moved, "flops": (10.0 if back else 4.0) * c["d"] * c["heads"] * pairs}


# ------------------------------------------------------------------------------------ 64 bits
def _exact_norm(s, c):
    x = s["x"].double()
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    h = (x - mean) / (var + EPS).sqrt()
    u = h if s["weight"] is None else torch.addcmul(s["bias"].double(), h, s["weight"].double())
    lead = (lambda t: t.double()) if c["mod"] == "token" else (lambda t: t.double().unsqueeze(1))
    a = None if s["scale"] is None else lead(s["scale"]) + 1
    return h, u, a, var, lead


def _exact_layer_norm(s, c):
    _, u, a, _, lead = _exact_norm(s, c)
    return {"y": u if a is None else torch.addcmul(lead(s["shift"]), u, a)}


def _exact_layer_norm_backward(s, c):
    h, u, a, var, _ = _exact_norm(s, c)
    dy, r = s["dy"].double(), {}
    if a is not None:
        r["dscale"], r["dshift"] = dy * u, dy
        if c["mod"] == "batch":
            r["dscale"], r["dshift"] = torch.einsum("bnc,bnc->bc", dy, u), dy.sum(1)
        dy = dy * a
    if c["affine"]:
        flat = dy.flatten(0, 1)
        r["dweight"], r["dbias"] = torch.einsum("nc,nc->c", flat, h.flatten(0, 1)), flat.sum(0)
        dy = dy * s["weight"].double()
    # the gradient less its parts along the ones and along h, whose squared length is c var / (var + eps)
    along = torch.einsum("bnc,bnc->bn", dy, h).unsqueeze(-1) / c["c"]
    r["dx"] = (dy - dy.mean(-1, keepdim=True) - along * h) / (var + EPS).sqrt()
    return r


def _exact_head(s, c, b, h):
    """(scaled products, derivative of the cap, scores) of one head in 64 bits, from the definition pair by pair."""
    q, k = s["q"][b, h].double(), s["k"][b, h * c["kv"] // c["heads"]].double()
    z = torch.mm(q, k.t()) / math.sqrt(c["d"])
    slope = None
    if c["cap"]:
        z = torch.tanh(z / c["cap"])
        slope = 1 - z.square()
        z = z * c["cap"]
    qe, ke, pe = (e[b] for e in _documents(c))
    seen = torch.zeros(c["nq"], c["nk"], dtype=torch.bool, device=GPU)
    for t in range(len(pe)):
        nq, nk = qe[t + 1] - qe[t], ke[t + 1] - ke[t]
        ahead = torch.arange(nk, device=GPU)[None] - (torch.arange(nq, device=GPU)[:, None] + nk - nq)  # of the query
        ok = (ahead <= 0) | (torch.arange(nk, device=GPU) < pe[t])[None] if c["causal"] else torch.ones_like(ahead, dtype=torch.bool)
        seen[qe[t]:qe[t + 1], ke[t]:ke[t + 1]] = ok
        if c["slopes"]:
            z[qe[t]:qe[t + 1], ke[t]:ke[t + 1]] -= 2.0 ** (-8.0 * (h + 1) / c["heads"]) * ahead.abs()
    return torch.where(seen, z, -math.inf), slope


def _exact_attention(s, c):
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=GPU)
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device=GPU)
    for b in range(c["batch"]):
        for h in range(c["heads"]):
            z, _ = _exact_head(s, c, b, h)
            lse[b, h] = torch.logsumexp(z, 1)
            p = torch.nan_to_num(torch.exp(z - lse[b, h][:, None]), nan=0.0)
            o[b, h] = torch.mm(p, s["v"][b, h * c["kv"] // c["heads"]].double())
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}


def _exact_attention_backward(s, c):
    r = {n: torch.zeros(s[n[1:]].shape, dtype=torch.float64, device=GPU) for n in ("dq", "dk", "dv")}
    for b in range(c["batch"]):
        for h in range(c["heads"]):
            at = h * c["kv"] // c["heads"]
            z, slope = _exact_head(s, c, b, h)
            p = torch.nan_to_num(torch.exp(z - s["lse"][b, h].double()[:, None]), nan=0.0)
            dy = s["dy"][b, h].double()
            r["dv"][b, at] += torch.mm(p.t(), dy)
            dp = torch.mm(dy, s["v"][b, at].double().t())
            ds = (dp - torch.einsum("nd,nd->n", dy, s["o"][b, h].double())[:, None]) * p / math.sqrt(c["d"])
            if slope is not None:
                ds = ds * slope
            r["dq"][b, h] = torch.mm(ds, s["k"][b, at].double())
            r["dk"][b, at] += torch.mm(ds.t(), s["q"][b, h].double())
    return r


def exact(case, seed):
    s = prepare(case, seed)
    return {"layer_norm": _exact_layer_norm, "layer_norm_backward": _exact_layer_norm_backward, "attention": _exact_attention,
            "attention_backward": _exact_attention_backward}[case["what"]](s, case)
