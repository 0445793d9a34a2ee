"""attention_block: linear, rotary, attention_layer and linear in a row, against the same steps in plain form, and captured."""
import pytest
import torch

import paper_2603_08982_amd as sv
from helpers import init_centroids
from projection_helpers import f64, linear64, rotary64
from workloads import budget_pairs

pytestmark = pytest.mark.gpu


def rand(*shape, seed=0, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def block(dtype, B=1, H=3, d=64, grid=(3, 5, 7), n_tail=6, c=80, Cq=4, Ck=9, norm="token", seed=0, gate="batch"):
    N = grid[0] * grid[1] * grid[2] + n_tail
    x = rand(B, N, c, seed=seed, dtype=dtype).cuda()
    w_qkv = rand(3 * H * d, c, seed=seed + 1, dtype=dtype, scale=c ** -0.5).cuda()
    b_qkv = rand(3 * H * d, seed=seed + 2, dtype=dtype, scale=0.1).cuda()
    w_out = rand(c, H * d, seed=seed + 3, dtype=dtype, scale=(H * d) ** -0.5).cuda()
    b_out = rand(c, seed=seed + 4, dtype=dtype, scale=0.1).cuda()
    g = rand(*((B, c) if gate == "batch" else (B, N, c)), seed=seed + 5, dtype=dtype).cuda()
    size = {"token": H * d, "head": d}[norm]
    weights = [(1 + 0.2 * rand(size, seed=seed + 6 + i)).to(dtype).cuda() for i in range(2)]
    sections = (10, 11, 11) if d == 64 else (22, 21, 21)
    kw = dict(inv_freq=sv.rotary_frequencies(sections), sections=sections, grid=grid, b_qkv=b_qkv, b_out=b_out, norm=norm,
              norm_weights=weights, gate=g, residual=x, n_tail=n_tail)
    return x, w_qkv, w_out, kw


def centroids(x, w_qkv, kw, H, d, Cq, Ck):
    """Starting centroids: rows of the rotated queries and keys, by the library's own calls."""
    B, N, _ = x.shape
    qkv, _ = sv.linear(x, w_qkv, kw["b_qkv"])
    q, k, v = qkv.view(B, N, 3, H, d).permute(2, 0, 3, 1, 4)
    q, k = sv.rotary([q, k], kw["inv_freq"], kw["sections"], grid=kw["grid"], n_tail=kw["n_tail"], norm=kw["norm"], weights=kw["norm_weights"])
    return q, k, v, init_centroids(q, Cq, 3, 0, kw["n_tail"]), init_centroids(k, Ck, 3, 1, kw["n_tail"])


@pytest.mark.parametrize("dtype,H,d,norm,B", [(torch.float32, 3, 64, "token", 1), (torch.bfloat16, 2, 128, "head", 2), (torch.bfloat16, 3, 64, "token", 1),
                                              (torch.float32, 2, 128, "head", 1)])
def test_block_against_plain_attention(dtype, H, d, norm, B):
    """With every key cluster routed (budget of all pairs) the layer is exact attention, which the plain steps in 64 bits compute from
    the block's inputs alone. A value passes five roundings to the type on its way (qkv, rotated, weights and values of the softmax,
    the layer's output), each half a step relative to values of its own size; the sum over the way is taken as 8 steps of the
    result's norm (bf16), and 2^-18 of it in fp32 (sums of up to 384 terms, half of them rounded each way)."""
    x, w_qkv, w_out, kw = block(dtype, H=H, d=d, norm=norm, B=B)
    N = x.shape[1]
    q, k, v, cq, ck = centroids(x, w_qkv, kw, H, d, 4, 9)
    y, r = sv.attention_block(x, w_qkv, w_out, cq.clone(), ck.clone(), 3, budget_pairs(1.0, N, N), **kw)
    qkv = linear64(x, w_qkv, kw["b_qkv"])[0].view(B, N, 3, H, d).permute(2, 0, 3, 1, 4)
    rot = [rotary64(t, kw["inv_freq"], kw["sections"], grid=kw["grid"], n_tail=kw["n_tail"], norm=norm, weight=w)[0]
           for t, w in zip(qkv[:2], kw["norm_weights"])]
    p = torch.softmax(rot[0] @ rot[1].transpose(2, 3) * d ** -0.5, -1)
    o = (p @ qkv[2]).transpose(1, 2).reshape(B, N, H * d)
    Y = (o @ f64(w_out).t() + f64(kw["b_out"])) * f64(kw["gate"])[:, None] + f64(x)
    off = float((f64(y) - Y).norm() / Y.norm())
    assert off <= (8 * 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -18), off


@pytest.mark.parametrize("dtype,top_p", [(torch.bfloat16, None), (torch.bfloat16, 0.7), (torch.float32, None)])
def test_block_equals_its_calls_in_a_row(dtype, top_p):
    """Strided views in place of dense tensors change nothing: the block gives the bits of linear, rotary, attention_layer on dense
    copies, and linear."""
    H, d = 3, 64
    x, w_qkv, w_out, kw = block(dtype, H=H, d=d, gate="token")
    B, N, _ = x.shape
    q, k, v, cq, ck = centroids(x, w_qkv, kw, H, d, 4, 9)
    budget = budget_pairs(0.3, N, N)
    cq1, ck1 = cq.clone(), ck.clone()
    y, r = sv.attention_block(x, w_qkv, w_out, cq1, ck1, 3, budget, top_p=top_p, **kw)
    O, r2 = sv.attention_layer(q, k, v.contiguous(), cq, ck, 3, budget, kw["n_tail"], top_p=top_p)
    y2, _ = sv.linear(O.transpose(1, 2).reshape(B, N, H * d), w_out, kw["b_out"], gate=kw["gate"], residual=x)
    assert torch.equal(r["O"], O) and torch.equal(y, y2)
    assert torch.equal(cq1, cq) and torch.equal(ck1, ck) and torch.equal(r["mask_bits"], r2["mask_bits"])


@pytest.mark.parametrize("token_order", [True, False])
def test_layer_writes_into_out(token_order):
    x, w_qkv, w_out, kw = block(torch.bfloat16)
    q, k, v, cq, ck = centroids(x, w_qkv, kw, 3, 64, 4, 9)
    N = x.shape[1]
    ref, _ = sv.attention_layer(q, k, v.contiguous(), cq.clone(), ck.clone(), 2, budget_pairs(0.3, N, N), kw["n_tail"])
    buf = torch.full((1, N, 3, 64 + 64), 5.0, dtype=torch.bfloat16, device="cuda")
    out = buf[..., :64].transpose(1, 2)
    O, _ = sv.attention_layer(q, k, v.contiguous(), cq.clone(), ck.clone(), 2, budget_pairs(0.3, N, N), kw["n_tail"], token_order=token_order, out=out)
    assert O is out and torch.equal(out, ref) and bool((buf[..., 64:] == 5).all())


def test_captured_block_replays_bit_exactly():
    H, d = 2, 128
    x, w_qkv, w_out, kw = block(torch.bfloat16, H=H, d=d)
    N = x.shape[1]
    _, _, _, cq0, ck0 = centroids(x, w_qkv, kw, H, d, 4, 9)
    budget = budget_pairs(0.3, N, N)
    xs, cq, ck = x.clone(), cq0.clone(), ck0.clone()
    kw["residual"] = xs

    def step():
        cq.copy_(cq0), ck.copy_(ck0)
        return sv.attention_block(xs, w_qkv, w_out, cq, ck, 3, budget, **kw)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    for r in range(3):
        xs.copy_(rand(*x.shape, seed=60 + r, dtype=x.dtype).cuda())
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, step())
