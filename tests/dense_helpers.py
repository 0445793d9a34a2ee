"""Plain 64-bit forms of the layer norm and of dense attention, with bounds on what fp32 arithmetic may be off by.

A bound is derived from the formula: each product or sum in fp32 is off by at most half a step of its result (U32 relative), a
sum by so many half steps of the sum of its terms' magnitudes as roundings lie on a term's way to the result, a value rounded to
bf16 on the way by half a step of that (UNIT), and the output by half a step of its type.
"""
import torch

from projection_helpers import U32, UNIT


def f64(t):
    return None if t is None else t.detach().double()


def close(got, want, bound, what=""):
    """got within `bound` and the output's own rounding of want, element by element; infinities and NaN where want has them."""
    unit = UNIT[got.dtype]
    g, want = f64(got), f64(want)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    off = (g - want).abs() - (bound * (1 + unit) + unit * want.abs() + 2.0 ** -126)
    ok = (off <= 0) | (g == want) | (g.isnan() & want.isnan())
    if not bool(ok.all()):
        i = int((~ok).flatten().nonzero()[0])
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.numel()} values outside; at {i}: {g.flatten()[i]} for "
                             f"{want.flatten()[i]} +- {(bound + torch.zeros_like(want)).flatten()[i]}")


# ----------------------------------------------------------------------------------- layer norm
# roundings on a term's way into a row's sum: at most 32 in a lane, 6 over the lanes, 16 over the waves, and the last products
ROW = 64 * U32
# and into a column's: the rows of a team (few hundred at most here), 32 runs of parts
COLUMN = 400 * U32


def spread(t, x):
    """A row for each batch entry, or token, over the tokens of x."""
    t = f64(t)
    return t if t.dim() == x.dim() else t.unsqueeze(-2)


def norm64(x, weight, bias, scale, shift, eps):
    """(y, bound, h, bound of h, root factor)"""
    X = f64(x)
    mean = X.mean(-1, keepdim=True)
    d = X - mean
    r = (d.square().mean(-1, keepdim=True) + eps).rsqrt()
    h = d * r
    # the mean's error shifts every value (and is second order in the squares); the squares' sum counts by half on the root
    eh = (ROW * X.abs().mean(-1, keepdim=True) + 2 * U32 * (X.abs() + mean.abs())) * r + (ROW + 4 * U32) * h.abs()
    u, e = h, eh
    if weight is not None:
        u, e = u * f64(weight), e * f64(weight).abs() + U32 * (u * f64(weight)).abs()
    if bias is not None:
        e = e + 2 * U32 * (u.abs() + f64(bias).abs())
        u = u + f64(bias)
    y = u
    if scale is not None:
        s = 1 + spread(scale, x)
        y, e = y * s, e * s.abs() + 4 * U32 * (u.abs() + (f64(bias).abs() if bias is not None else 0)) * (1 + s.abs())
    if shift is not None:
        e = e + 2 * U32 * (y.abs() + spread(shift, x).abs())
        y = y + spread(shift, x)
    return y, e, h, eh, r


def norm_backward64(dy, x, weight, bias, scale, eps):
    """{name: (value, bound)}"""
    _, _, h, eh, r = norm64(x, None, None, None, None, eps)
    D = f64(dy)
    w = f64(weight) if weight is not None else torch.ones(x.shape[-1], dtype=torch.float64, device=x.device)
    b = f64(bias) if bias is not None else torch.zeros_like(w)
    s = 1 + spread(scale, x) if scale is not None else torch.ones_like(D)
    du = D * s
    g = du * w
    mg, mgh = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    mag, magh = g.abs().mean(-1, keepdim=True), (g * h).abs().mean(-1, keepdim=True)
    egh = (g.abs() * eh).mean(-1, keepdim=True)
    e = r * (4 * U32 * g.abs() * (1 + 1 / s.abs().clamp(min=1e-3)) + ROW * mag + (ROW + 4 * U32) * (magh + mgh.abs()) * h.abs() + egh * h.abs() + mgh.abs() * eh
             + ROW * (g.abs() + mg.abs() + (h * mgh).abs()))
    out = {"dx": (r * (g - mg - h * mgh), e)}
    lead = tuple(range(x.dim() - 1))
    edu = 4 * U32 * D.abs() * (1 + s.abs())
    out["dweight"] = ((du * h).sum(lead), (COLUMN * (du * h).abs() + du.abs() * eh + edu * h.abs()).sum(lead))
    out["dbias"] = (du.sum(lead), (COLUMN * du.abs() + edu).sum(lead))
    u, eu = h * w + b, eh * w.abs() + 2 * U32 * ((h * w).abs() + b.abs())
    ds, es, eb = D * u, D.abs() * eu + COLUMN * D.abs() * ((h * w).abs() + b.abs()), COLUMN * D.abs()
    if scale is not None and scale.dim() == x.dim():
        out["dscale"], out["dshift"] = (ds, es), (D, 0 * eb)
    else:
        out["dscale"], out["dshift"] = (ds.sum(-2), es.sum(-2)), (D.sum(-2), eb.sum(-2))
    return out


# ------------------------------------------------------------------------------------ attention
def offsets_of(t, b, n):
    if t is None:
        return [0, n]
    return (t if t.dim() == 1 else t[b]).tolist()


def seen64(B, Nq, Nk, causal=False, prefix=None, q_offsets=None, k_offsets=None, device="cuda"):
    """(which key each query sees [B,Nq,Nk], query's position less the key's), pair by pair."""
    seen = torch.zeros(B, Nq, Nk, dtype=torch.bool, device=device)
    dist = torch.zeros(B, Nq, Nk, dtype=torch.float64, device=device)
    for b in range(B):
        qe, ke = offsets_of(q_offsets, b, Nq), offsets_of(k_offsets, b, Nk)
        for t in range(len(qe) - 1):
            n, m = qe[t + 1] - qe[t], ke[t + 1] - ke[t]
            p = 0 if prefix is None else int((prefix if prefix.dim() == 1 else prefix[b])[t])
            i, j = torch.arange(n, device=device)[:, None], torch.arange(m, device=device)[None]
            d = i + m - n - j
            ok = (d >= 0) | (j < p) if causal else torch.ones_like(d, dtype=torch.bool)
            seen[b, qe[t]:qe[t + 1], ke[t]:ke[t + 1]] = ok
            dist[b, qe[t]:qe[t + 1], ke[t]:ke[t + 1]] = d.double()
    return seen, dist


def scores64(q, k, scale, cap, slopes, **mask):
    """(s with -inf where unseen, bound of its error, 1 - tanh^2, what is seen [B,1,Nq,Nk])"""
    Q, K = f64(q), f64(k).repeat_interleave(q.shape[1] // k.shape[1], 1)
    d = q.shape[3]
    seen, dist = seen64(q.shape[0], q.shape[2], k.shape[2], device=q.device, **mask)
    seen = seen[:, None]
    s, e = Q @ K.transpose(2, 3) * scale, (d + 2) * U32 * abs(scale) * (Q.abs() @ K.abs().transpose(2, 3))
    keeps = torch.ones_like(s)
    if cap:
        th = torch.tanh(s / cap)
        # tanh from an exponential and a reciprocal, each off by a step or two of a number up to 2; slope at most 1
        s, keeps = cap * th, 1 - th * th
        e = e + (8 * U32 if q.dtype == torch.float32 else 16 * U32) * cap
    if slopes is not None:
        bias = f64(slopes)[:, None, None] * dist[:, None].abs()
        s, e = s - bias, e + 2 * U32 * (bias + s.abs())
    s = torch.where(seen, s, -torch.inf)
    return s, torch.where(seen, e, 0.0), keeps, seen


# Weights below the smallest normal number are taken as 0 (the exponential's and the matrix cores' results have no steps below
# it), which is off by less than it: a weight's own absolute error beside its relative one. Found by a case whose gradients were
# 1e-36: its 5 heads' weights of 2^-127 times queries of 1.4 lose 1.7e-38, which half steps of 2e-36 do not cover.
TINY = 2.0 ** -126


def safe(t):
    """Values of rows that nothing sees may be anything: they are taken out."""
    return torch.where(torch.isfinite(t), t, torch.zeros_like(t))


def attention64(q, k, v, scale=None, cap=None, slopes=None, **mask):
    """(o, bound, lse, bound). Rows of k and v that no query sees may hold anything."""
    scale = q.shape[3] ** -0.5 if scale is None else scale
    V = f64(v).repeat_interleave(q.shape[1] // k.shape[1], 1)
    s, es, _, seen = scores64(q, k, scale, cap, slopes, **mask)
    lse = torch.logsumexp(s, -1)
    some = seen.any(-1)
    some = some.expand(lse.shape)
    p = torch.where(seen, (s - torch.where(some, lse, 0.0)[..., None]).exp(), 0.0)
    big = torch.where(seen, s.abs(), 0.0).amax(-1, keepdim=True)
    # a weight: its exponent's error, that of the exponential, and the running maximum's; bf16: its rounding
    ep = es + 8 * U32 * (1 + big)
    unit = UNIT[q.dtype] if q.dtype == torch.bfloat16 else 0.0
    n = k.shape[2]
    o = p @ safe(V)
    el = (p * (ep + n * U32)).sum(-1)
    eo = (p * (ep + unit * (1 + ep) + (n + 8) * U32) + TINY * seen) @ safe(V).abs() + (el[..., None] + 4 * U32) * o.abs()
    return o, eo, torch.where(some, lse, -torch.inf), torch.where(some, 2 * el + 4 * U32 * (1 + lse.abs() + big[..., 0]), 0.0)


def attention_backward64(dy, q, k, v, o, lse, scale=None, cap=None, slopes=None, **mask):
    """{name: (value, bound)} by the formula, with the o and lse that are given."""
    scale = q.shape[3] ** -0.5 if scale is None else scale
    G, d = q.shape[1] // k.shape[1], q.shape[3]
    K, V = (safe(f64(t).repeat_interleave(G, 1)) for t in (k, v))
    Q, D, O = safe(f64(q)), f64(dy), f64(o)
    s, es, keeps, seen = scores64(q, k, scale, cap, slopes, **mask)
    some = seen.any(-1).expand(lse.shape)
    D, O = torch.where(some[..., None], D, 0.0), torch.where(some[..., None], O, 0.0)
    L = torch.where(some, f64(lse), 0.0)[..., None]
    p = torch.where(seen, (s - L).exp(), 0.0)
    big = torch.where(seen, s.abs() + L.abs(), 0.0)
    ep = es + 8 * U32 * (1 + big)
    dp, delta = D @ V.transpose(2, 3), (D * O).sum(-1, keepdim=True)
    edp = (d + 2) * U32 * (D.abs() @ V.abs().transpose(2, 3) + (D * O).abs().sum(-1, keepdim=True))
    ds = p * (dp - delta) * keeps
    # 1 - tanh^2 is off by a few steps of 1
    eds = ep * ds.abs() + p * (edp + 4 * U32 * (dp - delta).abs()) + (0.0 if not cap else 32 * U32) * (p * (dp - delta)).abs()
    unit = UNIT[q.dtype] if q.dtype == torch.bfloat16 else 0.0
    eds = eds * (1 + unit) + unit * ds.abs() + TINY * seen * (1 + (dp - delta).abs())
    epv = p * (ep + unit * (1 + ep)) + TINY * seen
    rows = q.shape[2] * G
    n = k.shape[2]

    def heads(t):
        return t.unflatten(1, (-1, G)).sum(2)

    eq = abs(scale) * ((eds + (n + 4) * U32 * ds.abs()) @ K.abs())
    ek = abs(scale) * heads((eds + (rows + 4) * U32 * ds.abs()).transpose(2, 3) @ Q.abs())
    ev = heads((epv + (rows + 4) * U32 * p).transpose(2, 3) @ D.abs())
    return {"dq": (scale * (ds @ K), eq), "dk": (scale * heads(ds.transpose(2, 3) @ Q), ek), "dv": (heads(p.transpose(2, 3) @ D), ev)}
