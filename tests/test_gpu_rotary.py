"""svgear_rotary and its backward pass against their formulas in 64 bits."""
import pytest
import torch

import paper_2603_08982_amd as sv
from projection_helpers import close, rotary64, rotary_backward64

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]
NAMES = {torch.bfloat16: "bf16", torch.float32: "f32"}


def rand(*shape, seed=0, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


# B, H, grid, first, n_tail, d, sections: one token, one pair, no rotation at all, part of a head, all of it; head counts around
# the 4 to 16 that a wave takes at a step, and up to several waves a token
CASES = [(1, 1, (1, 1, 1), 0, 0, 64, (0, 0, 1)), (2, 3, (2, 3, 5), 0, 0, 128, (22, 21, 21)), (1, 5, (3, 4, 5), 7, 9, 64, (10, 11, 11)),
         (2, 8, (1, 7, 9), 3, 1, 128, (0, 32, 32)), (1, 40, (2, 2, 3), 0, 0, 128, (22, 21, 21)), (1, 41, (2, 2, 2), 1, 3, 128, (16, 8, 8)),
         (1, 12, (4, 3, 3), 0, 2, 64, (0, 0, 0)), (3, 24, (1, 1, 7), 6, 4, 128, (8, 28, 28)), (1, 128, (1, 1, 3), 0, 1, 64, (8, 12, 11)),
         (1, 128, (1, 1, 2), 0, 0, 128, (3, 5, 7)), (1, 17, (1, 5, 5), 0, 0, 64, (16, 8, 8))]


def setup(case, dtype, norm, listed, seed=0):
    B, H, grid, first, n_tail, d, sections = case
    n = grid[0] * grid[1] * grid[2] - first
    kw = {"n_tail": n_tail, "norm": norm, "eps": 1e-6}
    if listed:
        g = torch.Generator().manual_seed(seed + 9)
        pos = torch.randint(-500, 200000, (B, n, 3), generator=g, dtype=torch.int32).cuda()
        kw["positions"] = pos if listed == "batch" else pos[0].contiguous()
    else:
        kw["grid"], kw["first"] = grid, first
    N = n + n_tail
    # a fused projection's output, so that heads and tokens are strided
    qkv = rand(B, N, 3, H, d, seed=seed, dtype=dtype, scale=1.5).cuda()
    q, k = qkv[:, :, 0].transpose(1, 2), qkv[:, :, 1].transpose(1, 2)
    size = {None: 0, "head": d, "token": H * d}[norm]
    weights = [1 + 0.3 * rand(size, seed=seed + 1 + i) for i in range(2)] if size else None
    weights = [w.to(dtype).cuda() for w in weights] if weights else None
    return q, k, sv.rotary_frequencies(sections), sections, weights, kw


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("norm", [None, "head", "token"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rotary_and_its_gradient(case, halves, norm, dtype):
    i = CASES.index(case)
    q, k, f, sections, weights, kw = setup(case, dtype, norm, [None, "shared", "batch"][i % 3], seed=100 * i)
    out = sv.rotary([q, k], f, sections, weights=weights, halves=halves, **kw)
    for x, y, w in zip((q, k), out, weights or (None, None)):
        assert y.is_contiguous()
        close(y, *rotary64(x, f, sections, weight=w, halves=halves, **kw), "y")
    B, H, N, d = q.shape
    grads = [rand(B, H, N, d, seed=100 * i + 50 + t, dtype=dtype).cuda() for t in range(2)]
    dx, dweight = sv.rotary_backward(grads, [q, k], f, sections, weights=weights, halves=halves, **kw)
    assert (dweight is None) == (norm is None)
    for t, (x, w) in enumerate(zip((q, k), weights or (None, None))):
        rdx, bdx, rdw, bdw = rotary_backward64(grads[t], x, f, sections, weight=w, halves=halves, **kw)
        close(dx[t], rdx, bdx, "dx")
        if norm is not None:
            close(dweight[t], rdw, bdw, "dweight")


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_many_tokens_share_the_sums_of_weights(dtype):
    """More tokens than the backward pass has workgroups: every token's part reaches dweight once."""
    for norm in ("head", "token"):
        q, k, f, sections, weights, kw = setup((1, 3, (13, 15, 17), 0, 20, 64, (10, 11, 11)), dtype, norm, None, seed=7)
        grads = [rand(*q.shape, seed=8 + t, dtype=dtype).cuda() for t in range(2)]
        dx, dweight = sv.rotary_backward(grads, [q, k], f, sections, weights=weights, **kw)
        for t, x in enumerate((q, k)):
            rdx, bdx, rdw, bdw = rotary_backward64(grads[t], x, f, sections, weight=weights[t], **kw)
            close(dx[t], rdx, bdx, "dx")
            close(dweight[t], rdw, bdw, "dweight")


def test_weightless_norms_one_tensor_and_no_weight_gradient():
    q, k, f, sections, weights, kw = setup((2, 5, (2, 3, 4), 0, 3, 128, (22, 21, 21)), torch.float32, "token", None)
    (y,) = sv.rotary([q], f, sections, **kw)
    close(y, *rotary64(q, f, sections, **kw))
    y = sv.rotary([q, k], f, sections, weights=[None, weights[1]], **kw)
    close(y[0], *rotary64(q, f, sections, **kw))
    close(y[1], *rotary64(k, f, sections, weight=weights[1], **kw))
    dx, dw = sv.rotary_backward([y[0]], [q], f, sections, want_dweight=False, **kw)
    assert dw is None
    rdx, bdx, _, _ = rotary_backward64(y[0], q, f, sections, **kw)
    close(dx[0], rdx, bdx)


@pytest.mark.parametrize("norm", [None, "head", "token"])
@pytest.mark.parametrize("halves", [False, True])
def test_in_place_equals_out_of_place(norm, halves):
    q, k, f, sections, weights, kw = setup((2, 9, (2, 5, 4), 0, 3, 128, (22, 21, 21)), torch.bfloat16, norm, None)
    ref = sv.rotary([q, k], f, sections, weights=weights, halves=halves, **kw)
    grads = [rand(*q.shape, seed=5 + t, dtype=torch.bfloat16).cuda() for t in range(2)]
    rdx, rdw = sv.rotary_backward(grads, [q, k], f, sections, weights=weights, halves=halves, **kw)
    kept = [g.clone() for g in grads]
    dx, dw = sv.rotary_backward(kept, [q, k], f, sections, weights=weights, halves=halves, out=kept, **kw)
    assert all(torch.equal(a, b) for a, b in zip(dx, rdx))
    assert dw is None or all(torch.equal(a, b) for a, b in zip(dw, rdw))
    out = sv.rotary([q, k], f, sections, weights=weights, halves=halves, out=[q, k], **kw)
    assert out[0] is q and torch.equal(q, ref[0]) and torch.equal(k, ref[1])


def test_single_tokens_into_a_cache_equal_the_whole_sequence():
    """Token by token, by `first` and by a position list, into the slots of a cache: the same bits as the whole at once, and the
    other slots untouched."""
    q, k, f, sections, weights, kw = setup((2, 6, (2, 3, 4), 0, 0, 128, (22, 21, 21)), torch.bfloat16, "token", None)
    ref = sv.rotary([q, k], f, sections, weights=weights, **kw)[1]
    cache = torch.full((2, 6, 40, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    kw.pop("grid"), kw.pop("first")
    for n in range(24):
        one = {"grid": (2, 3, 4), "first": n} if n % 2 else {"positions": torch.tensor([[n // 12, n // 4 % 3, n % 4]], dtype=torch.int32).cuda()}
        sv.rotary([k[:, :, n:n + 1]], f, sections, weights=weights[1:], out=[cache[:, :, 8 + n:9 + n]], **one, **kw)
    assert torch.equal(cache[:, :, 8:32], ref)
    assert bool((cache[:, :, :8] == 3).all()) and bool((cache[:, :, 32:] == 3).all())


def test_far_positions_keep_their_phase():
    """Positions up to 2^31 - 1 at frequency 1: the angle in fp64 is off by 2^-22 rad at most, far below an fp32 angle's 2^7."""
    pos = torch.tensor([[2 ** 31 - 1, 2 ** 30 + 1, -(2 ** 31)], [10 ** 9, 123456789, 7]], dtype=torch.int32).cuda()
    x = rand(1, 1, 2, 64, seed=1).cuda()
    f = torch.ones(32, dtype=torch.float64, device="cuda")
    (y,) = sv.rotary([x], f, (11, 11, 10), positions=pos)
    Y, b = rotary64(x, f, (11, 11, 10), positions=pos)
    close(y, Y, b + 2.0 ** -22 * 4)


def test_infinities_and_zero_rows():
    """A token of zeros gives zeros, one with an infinity spoils only itself, and what is not rotated is copied, infinities too."""
    q, _, f, sections, weights, kw = setup((1, 5, (2, 3, 4), 0, 4, 128, (10, 10, 10)), torch.float32, None, None)
    q[0, 2, 25, 3] = float("inf")   # a text token
    q[0, 1, 5, 100] = float("-inf")  # beyond the rotated pairs
    for halves in (False, True):
        (y,) = sv.rotary([q], f, sections, halves=halves, **kw)
        bad = ~y.isfinite()
        assert int(bad.sum()) == 2 and y[0, 2, 25, 3] == float("inf") and y[0, 1, 5, 100] == float("-inf")
    q[0, 2, 25, 3] = q[0, 1, 5, 100] = 1.0
    for norm in ("head", "token"):
        kw["norm"] = norm
        q[0, :, 3] = 0.0
        q[0, 0, 4, 1] = float("nan")
        (y,) = sv.rotary([q], f, sections, **kw)
        assert bool((y[0, :, 3] == 0).all())
        bad = y.isnan().any(-1)[0]  # [heads, tokens]
        assert int(bad.sum()) == (1 if norm == "head" else 5) and bool(bad[:, 4].any())


def test_gradients_against_differences():
    """Central differences of sum(y c), fp32, h = 2^-6: rounding and third derivatives stay under 1e-3 of the terms' magnitudes."""
    q, k, f, sections, weights, kw = setup((1, 6, (2, 3, 4), 0, 3, 64, (10, 11, 11)), torch.float32, "token", None)
    c = rand(*q.shape, seed=2).cuda()
    dx, dw = sv.rotary_backward([c], [q], f, sections, weights=weights[:1], **kw)
    loss = lambda x, w: (sv.rotary([x], f, sections, weights=[w], **kw)[0].double() * c.double()).sum()
    h = 2.0 ** -6
    for name, got, t in (("dx", dx[0], rand(*q.shape, seed=3).cuda()), ("dweight", dw[0], rand(*weights[0].shape, seed=4).cuda())):
        up = (q + h * t, weights[0]) if name == "dx" else (q, weights[0] + h * t)
        down = (q - h * t, weights[0]) if name == "dx" else (q, weights[0] - h * t)
        diff = float((loss(*up) - loss(*down)) / (2 * h))
        terms = got.double() * t.double()
        assert abs(diff - float(terms.sum())) <= 1e-3 * float(terms.abs().sum()), name


def test_captured_and_replayed():
    q, k, f, sections, weights, kw = setup((2, 6, (2, 5, 7), 0, 3, 128, (22, 21, 21)), torch.bfloat16, "token", None)
    qs, ks = q.clone(), k.clone()
    grads = [rand(*q.shape, seed=3 + t, dtype=torch.bfloat16).cuda() for t in range(2)]

    def step(a, b):
        y = sv.rotary([a, b], f, sections, weights=weights, **kw)
        dx, dw = sv.rotary_backward(grads, [a, b], f, sections, weights=weights, **kw)
        return [*y, *dx, *dw]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(qs, ks)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(qs, ks)
    for r in range(3):
        a, b = (rand(*q.shape, seed=20 + 2 * r + t, dtype=torch.bfloat16).cuda() for t in range(2))
        qs.copy_(a), ks.copy_(b)
        graph.replay()
        ref = step(a, b)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, ref))


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_a_cache_of_more_than_4_gib(dtype):
    """Heads that lie more than 2^31 elements apart, forward and backward."""
    far, d, n = (1 << 31) + 64, 64, 5
    x = rand(1, 2, n, d, seed=1, dtype=dtype).cuda()
    f, sections = sv.rotary_frequencies((10, 11, 11)), (10, 11, 11)
    kw = {"grid": (1, 1, n), "norm": "head"}
    w = rand(d, seed=2, dtype=dtype).cuda()
    cache = torch.empty(far + n * d, dtype=dtype, device="cuda").as_strided((1, 2, n, d), (2 * far, far, d, 1))
    sv.rotary([x], f, sections, weights=[w], out=[cache], **kw)
    close(cache, *rotary64(x, f, sections, weight=w, **kw))
    g = rand(1, 2, n, d, seed=3, dtype=dtype).cuda()
    dx, dw = sv.rotary_backward([g], [cache], f, sections, weights=[w], **kw)
    rdx, bdx, rdw, bdw = rotary_backward64(g, cache, f, sections, weight=w, **kw)
    close(dx[0], rdx, bdx)
    close(dw[0], rdw, bdw)


def test_calls_on_two_streams_at_once():
    a = setup((2, 40, (1, 5, 30), 0, 7, 128, (22, 21, 21)), torch.bfloat16, "token", None, seed=30)
    b = setup((1, 5, (3, 20, 10), 0, 0, 64, (8, 12, 11)), torch.float32, "head", "batch", seed=40)

    def step(q, k, f, sections, weights, kw):
        y = sv.rotary([q, k], f, sections, weights=weights, **kw)
        dx, dw = sv.rotary_backward(y, [q, k], f, sections, weights=weights, **kw)
        return [*y, *dx, *dw]

    ra, rb = step(*a), step(*b)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(3):
        with torch.cuda.stream(s1):
            got.append((step(*a), ra))
        with torch.cuda.stream(s2):
            got.append((step(*b), rb))
    torch.cuda.synchronize()
    for g, r in got:
        assert all(torch.equal(u, v) for u, v in zip(g, r))


def test_strides_of_single_elements_do_not_matter():
    """[1,H,1,d] views whose batch and token strides are no whole chunks."""
    x = rand(1, 5, 1, 64, seed=1).cuda()
    odd = torch.empty(5 * 64 + 64, device="cuda").as_strided((1, 5, 1, 64), (7, 64, 3, 1))
    odd.copy_(x)
    f, sections = sv.rotary_frequencies((10, 11, 11)), (10, 11, 11)
    kw = {"grid": (3, 4, 5), "first": 33, "norm": "token"}
    ref, got = sv.rotary([x], f, sections, **kw)[0], sv.rotary([odd], f, sections, out=[odd], **kw)[0]
    assert torch.equal(ref, got)


@pytest.mark.parametrize("norm", [None, "head", "token"])
def test_more_tokens_than_a_launch_has_threads_for(norm):
    """2^26 tokens are 2^32 threads. Shares of them, anywhere, come to what a call of their own gives."""
    n, d, sections = (1 << 26) + 9, 64, (10, 11, 11)
    x = rand(1, 1, 1 << 14, d, seed=1, dtype=torch.bfloat16).cuda().repeat(1, 1, (n >> 14) + 1, 1)[:, :, :n]
    x[:, :, -9:] = 2.0
    f, grid = sv.rotary_frequencies(sections), (n, 1, 1)
    weights = [rand(64, seed=2, dtype=torch.bfloat16).cuda()] if norm else None
    y, = sv.rotary([x], f, sections, grid=grid, norm=norm, weights=weights)
    dx, _ = sv.rotary_backward([x], [x] if norm else None, f, sections, grid=grid, norm=norm, weights=weights, want_dweight=False)
    for at in (0, n // 2 + 1, (1 << 26) - 50, n - 100):
        part = x[:, :, at:at + 100]
        want, = sv.rotary([part], f, sections, grid=grid, first=at, norm=norm, weights=weights)
        assert torch.equal(y[:, :, at:at + 100], want), at
        want, _ = sv.rotary_backward([part], [part] if norm else None, f, sections, grid=grid, first=at, norm=norm, weights=weights,
                                     want_dweight=False)
        assert torch.equal(dx[0][:, :, at:at + 100], want[0]), at
