"""Plain 64-bit forms of linear and rotary (CPU, elementwise formulas) with bounds on what fp32 arithmetic may be off by.

A bound is derived from the formula: each product or sum in fp32 is off by at most half a step of its result (U32 relative), a
sum of n terms by n U32 of the sum of the terms' magnitudes in whatever order, and the one rounding to the output's type by
half a step of it (UNIT).
"""
import math

import torch

U32 = 2.0 ** -24
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
# exp, erfc and sin of the device's library are good to a few steps; an argument up to 2^6, itself rounded, puts 2^6 steps
# on an exponential
ACT = 2.0 ** 7 * U32


def f64(t):
    return None if t is None else t.detach().cpu().double()


def act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope64(z, act):
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad(act64(z, act).sum() if act != "none" else z.sum(), z)[0]


def gate64(gate, y):
    """The gate spread over the tokens of [.., N, d_out]."""
    g = f64(gate)
    return torch.ones(1, dtype=torch.float64) if g is None else g if g.dim() == y.dim() else g.unsqueeze(-2)


def linear64(x, w, bias=None, act="none", gate=None, residual=None):
    """(y, z, bound of y before its rounding, bound of z before its rounding)."""
    X, W = f64(x), f64(w)
    K = X.shape[-1]
    z, mag = X @ W.t(), X.abs() @ W.abs().t()
    if bias is not None:
        z, mag = z + f64(bias), mag + f64(bias).abs()
    dz = (K + 2) * U32 * mag
    a = act64(z, act)
    # no activation here is steeper than 1.13
    da = 1.13 * dz + (0.0 if act == "none" else ACT) * z.abs()
    g = gate64(gate, z)
    y, dy = a * g, da * g.abs() + 2 * U32 * (a * g).abs()
    if residual is not None:
        y = y + f64(residual)
        dy = dy + 2 * U32 * (y.abs() + (a * g).abs())
    return y, z, dy, dz


def linear_backward64(dy, x, w, pre, act="none", gate=None, unit=U32):
    """{name: (value, bound before the output's rounding)}; unit: half a step of what dz is rounded to for the products."""
    D = f64(dy)
    z = f64(pre) if pre is not None else torch.zeros_like(D)
    a, sl, g = act64(z, act), slope64(z, act), gate64(gate, D)
    dz = D * sl * g
    # the slope is made of terms up to 1 + |z| in size
    ddz = (0.0 if act == "none" else ACT * (1 + z.abs())) * (D * g).abs() + 3 * U32 * dz.abs()
    da, dda = D * a, (0.0 if act == "none" else ACT) * (D * z).abs() + 2 * U32 * (D * a).abs()
    O = D.shape[-1]
    M = D.numel() // O
    r = {"dbias": (dz.reshape(M, O).sum(0), (ddz + M * U32 * dz.abs()).reshape(M, O).sum(0))}
    if gate is not None:
        if gate.dim() == D.dim():
            r["dgate"] = (da, dda)
        else:
            n = D.shape[-2]
            r["dgate"] = (da.sum(-2), (dda + n * U32 * da.abs()).sum(-2))
    rounded = ddz * (1 + unit) + unit * dz.abs()  # dz as the products see it
    if w is not None:
        W = f64(w)
        r["dx"] = (dz @ W, (rounded + (O + 2) * U32 * dz.abs()) @ W.abs())
    if x is not None:
        X = f64(x).reshape(M, -1)
        z2, e2 = dz.reshape(M, O), (rounded + (M + 2) * U32 * dz.abs()).reshape(M, O)
        r["dw"] = (z2.t() @ X, e2.t() @ X.abs())
    return r


def close(got, want, bound, what=""):
    """got within `bound` and the output's own rounding of want, element by element."""
    unit = UNIT[got.dtype]
    g = f64(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    # the smallest normal number: below it the steps no longer shrink
    off = (g - want).abs() - (bound * (1 + unit) + unit * want.abs() + 2.0 ** -126)
    ok = (off <= 0) | (g == want) | (g.isnan() & want.isnan())
    if not bool(ok.all()):
        i = int((~ok).flatten().nonzero()[0])
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.numel()} values outside; at {i}: {g.flatten()[i]} for "
                             f"{want.flatten()[i]} +- {(bound + torch.zeros_like(want)).flatten()[i]}")


# ------------------------------------------------------------------------------------- rotary
def angles64(inv_freq, sections, grid, first, positions, n_rot, B):
    f = f64(inv_freq)
    if positions is not None:
        pos = f64(positions)
        pos = pos[None].expand(B, -1, -1) if pos.dim() == 2 else pos
    else:
        i = torch.arange(first, first + n_rot)
        pos = torch.stack([i // (grid[1] * grid[2]), i // grid[2] % grid[1], i % grid[2]], 1).double()[None].expand(B, -1, -1)
    axis = torch.tensor([0] * sections[0] + [1] * sections[1] + [2] * sections[2], dtype=torch.long)
    return pos[:, :, axis] * f


def turn64(x, angle, n_rot, halves, sign=1.0):
    """x [B,H,N,d] with the pairs of its first n_rot tokens turned, and the magnitudes that went into each element."""
    y, mag = x.clone(), x.abs().clone()
    P = angle.shape[-1]
    c, s = angle.cos()[:, None], (sign * angle).sin()[:, None]
    v = x[:, :, :n_rot]
    i = torch.arange(P)
    ia, ib = (i, i + P) if halves else (2 * i, 2 * i + 1)
    a, b = v[..., ia], v[..., ib]
    y[:, :, :n_rot, ia], y[:, :, :n_rot, ib] = a * c - b * s, a * s + b * c
    mag[:, :, :n_rot, ia] = mag[:, :, :n_rot, ib] = a.abs() + b.abs()
    return y, mag


def norm64(x, norm, eps):
    over = (3,) if norm == "head" else (1, 3)
    return torch.rsqrt(x.square().mean(over, keepdim=True) + eps)


def weight64(w, norm, x):
    if w is None:
        return torch.ones(1, dtype=torch.float64)
    return f64(w) if norm == "head" else f64(w).view(x.shape[1], 1, x.shape[3])


# steps of fp32 that a rotated value may be off by, of the magnitudes of its pair: a mean of squares summed in chains of at most
# 128 per lane with half its error on the root, the root, three factors, a sine whose argument is off by pi steps, four products
TURN = 128 * U32


def rotary64(x, inv_freq, sections, grid=None, first=0, positions=None, n_tail=0, norm=None, weight=None, eps=1e-6, halves=False):
    X = f64(x)
    n_rot = X.shape[2] - n_tail
    u = X if norm is None else X * norm64(X, norm, eps) * weight64(weight, norm, X)
    y, mag = turn64(u, angles64(inv_freq, sections, grid, first, positions, n_rot, X.shape[0]), n_rot, halves)
    return y, TURN * mag


def rotary_backward64(dy, x, inv_freq, sections, grid=None, first=0, positions=None, n_tail=0, norm=None, weight=None, eps=1e-6,
                      halves=False):
    """(dx, its bound, dweight or None, its bound)"""
    D = f64(dy)
    n_rot = D.shape[2] - n_tail
    du, mag = turn64(D, angles64(inv_freq, sections, grid, first, positions, n_rot, D.shape[0]), n_rot, halves, -1.0)
    if norm is None:
        return du, TURN * mag, None, None
    X = f64(x)
    f, w = norm64(X, norm, eps), weight64(weight, norm, X)
    over = (3,) if norm == "head" else (1, 3)
    count = X.shape[3] * (1 if norm == "head" else X.shape[1])
    g, gmag = du * w, mag * w.abs()
    dot, dmag = (g * X).sum(over, keepdim=True) / count, (gmag * X.abs()).sum(over, keepdim=True) / count
    dx = f * (g - X * f * f * dot)
    # the two terms and the sum behind the second one, each off by at most 3 TURN of its magnitudes
    bdx = 3 * TURN * f * (gmag + X.abs() * f * f * dmag)
    t, tm = du * X * f, mag * (X * f).abs()
    axes = (0, 1, 2) if norm == "head" else (0, 2)
    n = X.numel() // X.shape[3] // (1 if norm == "head" else X.shape[1])
    dw, bdw = t.sum(axes), (2 * TURN + n * U32) * tm.sum(axes)
    return dx, bdx, dw.flatten(), bdw.flatten()
