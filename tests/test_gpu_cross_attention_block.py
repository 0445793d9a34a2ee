"""cross_attention_block and its backward pass: against the same in 64 bits, against its calls in a row, and captured."""
import pytest
import torch

import paper_2603_08982_amd as sv

pytestmark = pytest.mark.gpu

B, N, M, C, CT, H, HK, D = 2, 203, 77, 192, 136, 4, 2, 64


def make(dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = lambda *s, scale=1.0, mean=0.0: (torch.randn(*s, generator=g, device="cuda") * scale + mean).to(dtype)
    a = {"x": t(B, N, C), "context": t(B, M, CT), "w_q": t(H * D, C, scale=C ** -0.5), "w_kv": t(2 * HK * D, CT, scale=CT ** -0.5),
         "w_out": t(C, H * D, scale=(H * D) ** -0.5), "norm_weight": t(C, scale=0.2, mean=1.0), "norm_bias": t(C, scale=0.2),
         "scale": t(B, C, scale=0.2), "shift": t(B, C, scale=0.2), "b_q": t(H * D, scale=0.1), "b_kv": t(2 * HK * D, scale=0.1),
         "b_out": t(C, scale=0.1), "gate": t(B, C), "residual": t(B, N, C)}
    lengths = torch.tensor([M, 31], dtype=torch.int32, device="cuda")
    a["context"][1, 31:] = 100.0  # padding, which must not matter
    return a, lengths, t(B, N, C)


def plain64(a, lengths):
    """The block in 64 bits with torch's graph of gradients; arguments as leaves."""
    p = {n: v.detach().double().requires_grad_(True) for n, v in a.items()}
    x = p["x"]
    h = (x - x.mean(-1, keepdim=True)) * (x.var(-1, correction=0, keepdim=True) + 1e-6).rsqrt()
    h = (h * p["norm_weight"] + p["norm_bias"]) * (1 + p["scale"][:, None]) + p["shift"][:, None]
    q = (h @ p["w_q"].t() + p["b_q"]).view(B, N, H, D).transpose(1, 2)
    k, v = (p["context"] @ p["w_kv"].t() + p["b_kv"]).view(B, M, 2, HK, D).permute(2, 0, 3, 1, 4)
    k, v = (t.repeat_interleave(H // HK, 1) for t in (k, v))
    s = q @ k.transpose(2, 3) * D ** -0.5
    s = s.masked_fill(torch.arange(M, device="cuda") >= lengths[:, None, None, None], -torch.inf)
    o = (s.softmax(-1) @ v).transpose(1, 2).reshape(B, N, H * D)
    y = p["residual"] + p["gate"][:, None] * (o @ p["w_out"].t() + p["b_out"])
    return y, p


def run(a, lengths, dy=None):
    kw = {n: a[n] for n in a if n not in ("x", "context", "w_q", "w_kv", "w_out")}
    y, kept = sv.cross_attention_block(a["x"], a["context"], a["w_q"], a["w_kv"], a["w_out"], H, lengths=lengths, saved=dy is not None, **kw)
    return (y, None) if dy is None else (y, sv.cross_attention_block_backward(dy, kept))


# A chain of four calls rounds seven (forward) to fifteen (gradients) tensors by half a step of 2^-8 or 2^-24 each; roundings are
# independent, so norms of the errors add as squares at most: sqrt(15) 2^-8 = 0.016, and with factors of up to 2 between them 0.03. In
# fp32 sums of 2,000 terms add to it: 100 steps.
TOL = {torch.bfloat16: 0.03, torch.float32: 100 * 2.0 ** -24}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_against_64_bits(dtype):
    a, lengths, dy = make(dtype)
    y, grads = run(a, lengths, dy)
    want, leaves = plain64(a, lengths)
    rel = lambda got, ref: ((got.double() - ref).norm() / ref.norm()).item()
    assert rel(y, want.detach()) < TOL[dtype]
    want.backward(dy.double())
    assert set(grads) == set(a) - {"residual"}
    for n, g in grads.items():
        assert g.shape == a[n].shape and rel(g, leaves[n].grad) < TOL[dtype], (n, rel(g, leaves[n].grad))
    assert (grads["context"][1, 31:] == 0).all()
    assert torch.equal(run(a, lengths)[0], y)


def test_calls_in_a_row():
    a, lengths, dy = make(torch.bfloat16, 1)
    y, _ = run(a, lengths)
    h = sv.layer_norm(a["x"], a["norm_weight"], a["norm_bias"], scale=a["scale"], shift=a["shift"])
    q = sv.linear(h, a["w_q"], a["b_q"])[0].view(B, N, H, D).transpose(1, 2)
    kv = sv.linear(a["context"], a["w_kv"], a["b_kv"])[0].view(B, M, 2, HK, D)
    offsets = torch.stack([torch.zeros_like(lengths), lengths], 1)
    o, _ = sv.attention(q, kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2), k_offsets=offsets)
    again, _ = sv.linear(o.transpose(1, 2).reshape(B, N, H * D), a["w_out"], a["b_out"], gate=a["gate"], residual=a["residual"])
    assert torch.equal(again, y)


def test_least_arguments():
    a, _, dy = make(torch.bfloat16, 2)
    y, kept = sv.cross_attention_block(a["x"], a["context"], a["w_q"], a["w_kv"], a["w_out"], H, saved=True)
    grads = sv.cross_attention_block_backward(dy, kept)
    assert set(grads) == {"x", "context", "w_q", "w_kv", "w_out"} and all(torch.isfinite(g).all() for g in grads.values())


def test_captured():
    a, lengths, dy = make(torch.bfloat16, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(a, lengths, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, grads = run(a, lengths, dy)
    for _ in range(3):
        a["x"].copy_(torch.randn_like(a["x"]))
        graph.replay()
        want, ref = run(a, lengths, dy)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and all(torch.equal(grads[n], ref[n]) for n in ref)


@pytest.mark.parametrize("change", [{"lengths": torch.zeros(2, dtype=torch.int64)}, {"heads": 5}, {"w_kv": (100, CT)}, {"context": (3, M, CT)}], ids=str)
def test_refuses(change):
    a, lengths, _ = make(torch.bfloat16, 4)
    kw = {"heads": H, "lengths": lengths, **{n: a[n] for n in ("x", "context", "w_q", "w_kv", "w_out")}}
    for n, v in change.items():
        kw[n] = torch.zeros(*v, dtype=torch.bfloat16, device="cuda") if isinstance(v, tuple) else v.cuda() if isinstance(v, torch.Tensor) else v
    with pytest.raises(sv.SvgearError):
        sv.cross_attention_block(**kw)


@pytest.mark.parametrize("without", [["scale"], ["shift"], ["scale", "norm_weight", "norm_bias", "gate"], ["b_q", "b_kv", "b_out"]], ids=str)
def test_gradients_of_what_is_given(without):
    """Every argument that is given has its gradient, a shift without a scale too."""
    a, lengths, dy = make(torch.float32, 5)
    full = dict(a)
    for n in without:
        del a[n]
        full[n] = torch.ones_like(full[n]) if n in ("norm_weight", "gate") else torch.zeros_like(full[n])
    y, grads = run(a, lengths, dy)
    want, leaves = plain64(full, lengths)
    want.backward(dy.double())
    assert set(grads) == set(a) - {"residual"}
    for n, g in grads.items():
        assert g.shape == a[n].shape and (g.double() - leaves[n].grad).norm() < TOL[torch.float32] * leaves[n].grad.norm(), n
