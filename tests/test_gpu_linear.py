"""svgear_linear and its backward pass against their formulas in 64 bits."""
import pytest
import torch

import paper_2603_08982_amd as sv
from projection_helpers import UNIT, close, linear64, linear_backward64

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]
NAMES = {torch.bfloat16: "bf16", torch.float32: "f32"}


def rand(*shape, seed=0, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def inputs(dtype, B, N, k, o, bias, gate, residual, seed):
    lead = (B, N) if B else (N,)
    x = rand(*lead, k, seed=seed, dtype=dtype).cuda()
    w = rand(o, k, seed=seed + 1, dtype=dtype, scale=k ** -0.5).cuda()
    b = rand(o, seed=seed + 2, dtype=dtype).cuda() if bias else None
    shape = {"none": None, "batch": (*lead[:-1], o), "token": (*lead, o)}[gate]
    g = rand(*shape, seed=seed + 3, dtype=dtype).cuda() if shape else None
    r = rand(*lead, o, seed=seed + 4, dtype=dtype).cuda() if residual else None
    return x, w, b, g, r


# (B, N, d_in, d_out): single rows, sizes around the tiles' and the steps' (32, 64, 128, 256), primes, one of everything,
# batches that divide tiles unevenly, long contractions with few rows and few columns
SIZES = [(1, 1, 1, 1), (1, 1, 256, 512), (3, 1, 640, 96), (1, 2, 5000, 72), (2, 7, 64, 64), (1, 16, 128, 80), (1, 17, 72, 130),
         (1, 33, 200, 31), (0, 31, 8, 257), (1, 128, 128, 128), (1, 129, 136, 136), (2, 100, 1003, 67), (3, 85, 131, 259),
         (1, 256, 64, 256), (1, 257, 320, 264), (1, 700, 96, 520), (2, 300, 4100, 40), (1, 64, 8200, 16), (5, 3, 77, 1)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_of_every_size(size, dtype):
    i = SIZES.index(size)
    act = ["none", "silu", "gelu", "gelu_tanh"][i % 4]
    gate = ["none", "batch", "token"][i % 3]
    x, w, b, g, r = inputs(dtype, *size, bias=i % 5 != 0, gate=gate, residual=i % 2 == 0, seed=10 * i)
    y, pre = sv.linear(x, w, b, act=act, gate=g, residual=r, want_pre=True)
    Y, Z, by, bz = linear64(x, w, b, act, g, r)
    close(pre, Z, bz, "pre")
    close(y, Y, by, "y")


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("rows", [2, 150])
def test_every_epilogue(rows, act, dtype):
    for bias in (False, True):
        for gate in ("none", "batch", "token"):
            for residual in (False, True):
                x, w, b, g, r = inputs(dtype, 2, rows, 96, 200, bias, gate, residual, seed=3)
                y, pre = sv.linear(x, w, b, act=act, gate=g, residual=r)
                assert pre is None
                Y, _, by, _ = linear64(x, w, b, act, g, r)
                close(y, Y, by, f"bias={bias} gate={gate} residual={residual}")


# an output of 17 x 17 tiles of 256 in each of the three products, with edges in every direction, and contractions of one to
# several steps, with an odd end
WIDE = [(1, 4099, 72, 4104), (1, 4099, 200, 4104), (1, 4099, 4104, 136), (2, 75, 4104, 4104), (3, 1367, 331, 4104), (1, 4099, 64, 4099)]


@pytest.mark.parametrize("size", WIDE, ids=str)
def test_large_outputs(size):
    i = WIDE.index(size)
    x, w, b, g, r = inputs(torch.bfloat16, *size, bias=True, gate=["batch", "token"][i % 2], residual=True, seed=200 + i)
    y, pre = sv.linear(x, w, b, act="silu", gate=g, residual=r, want_pre=True)
    Y, Z, by, bz = linear64(x, w, b, "silu", g, r)
    close(pre, Z, bz, "pre")
    close(y, Y, by, "y")
    dy = rand(*pre.shape, seed=300 + i, dtype=torch.bfloat16).cuda()
    got = sv.linear_backward(dy, x, w, pre=pre, act="silu", gate=g, want=["dx", "dw", "dbias", "dgate"])
    ref = linear_backward64(dy, x, w, pre, "silu", g, UNIT[torch.bfloat16])
    for name in got:
        close(got[name], *ref[name], name)


# products of up to 32 rows by so many columns that they take more than one tile of 64 x 64 on a compute unit: of the forward
# pass, of dx, and of dw (24 outputs)
FLAT = [(1, 9, 72, 17000), (1, 32, 200, 17003), (2, 15, 17000, 72), (1, 3, 17003, 24), (1, 33, 17000, 40), (1, 300, 17000, 24)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("size", FLAT, ids=str)
def test_few_rows_of_many_columns(size, dtype):
    i = FLAT.index(size)
    x, w, b, g, r = inputs(dtype, *size, bias=True, gate=["batch", "token"][i % 2], residual=True, seed=400 + i)
    y, pre = sv.linear(x, w, b, act="silu", gate=g, residual=r, want_pre=True)
    Y, Z, by, bz = linear64(x, w, b, "silu", g, r)
    close(pre, Z, bz, "pre")
    close(y, Y, by, "y")
    y, _ = sv.linear(x, w, b, gate=g, residual=r)
    Y, _, by, _ = linear64(x, w, b, "none", g, r)
    close(y, Y, by, "y without activation")
    dy = rand(*pre.shape, seed=500 + i, dtype=dtype).cuda()
    got = sv.linear_backward(dy, x, w, pre=pre, act="silu", gate=g, want=["dx", "dw", "dbias", "dgate"])
    ref = linear_backward64(dy, x, w, pre, "silu", g, UNIT[dtype])
    for name in got:
        close(got[name], *ref[name], name)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward_of_every_size(size, dtype):
    i = SIZES.index(size)
    act = ["silu", "none", "gelu_tanh", "gelu"][i % 4]
    gate = ["token", "none", "batch"][i % 3]
    x, w, b, g, _ = inputs(dtype, *size, bias=True, gate=gate, residual=False, seed=10 * i)
    _, pre = sv.linear(x, w, b, act=act, gate=g, want_pre=True)
    dy = rand(*pre.shape, seed=77 + i, dtype=dtype).cuda()
    want = ["dx", "dw", "dbias"] + (["dgate"] if g is not None else [])
    got = sv.linear_backward(dy, x, w, pre=pre, act=act, gate=g, want=want)
    ref = linear_backward64(dy, x, w, pre, act, g, UNIT[dtype])
    assert set(got) == set(want)
    for name in want:
        close(got[name], ref[name][0], ref[name][1], name)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("name", ["dx", "dw", "dbias", "dgate"])
def test_each_gradient_alone(name, dtype):
    x, w, b, g, _ = inputs(dtype, 2, 75, 104, 72, True, "batch", False, seed=5)
    _, pre = sv.linear(x, w, b, act="silu", gate=g, want_pre=True)
    dy = rand(*pre.shape, seed=9, dtype=dtype).cuda()
    got = sv.linear_backward(dy, x if name == "dw" else None, w if name == "dx" else None, pre=pre, act="silu", gate=g, want=[name])
    ref = linear_backward64(dy, x, w, pre, "silu", g, UNIT[dtype])[name]
    close(got[name], *ref, name)


def test_gradients_against_differences():
    """Directional derivatives of sum(y c) by the backward pass against central differences of the forward one, fp32. A difference
    over 2h loses U32 |loss terms| / h to rounding and h^2 to the third derivative; h = 2^-6 keeps both under 1e-3 of the sum of
    the terms' magnitudes."""
    x, w, b, g, r = inputs(torch.float32, 2, 40, 72, 56, True, "batch", True, seed=21)
    c = rand(2, 40, 56, seed=22).cuda()

    def loss(x, w, b, g):
        return (sv.linear(x, w, b, act="gelu_tanh", gate=g, residual=r)[0].double() * c.double()).sum()

    _, pre = sv.linear(x, w, b, act="gelu_tanh", gate=g, want_pre=True)
    got = sv.linear_backward(c, x, w, pre=pre, act="gelu_tanh", gate=g, want=["dx", "dw", "dbias", "dgate"])
    args, h = [x, w, b, g], 2.0 ** -6
    for k, name in enumerate(["dx", "dw", "dbias", "dgate"]):
        t = rand(*args[k].shape, seed=30 + k).cuda() * (0.2 if k == 1 else 1.0)
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + h * t, args[k] - h * t
        diff = float((loss(*up) - loss(*down)) / (2 * h))
        terms = got[name].double() * t.double()
        assert abs(diff - float(terms.sum())) <= 1e-3 * float(terms.abs().sum()), name


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_strides_and_odd_addresses(dtype):
    """Inputs that are slices of larger tensors, at any alignment, and batches that are not one run of rows; rows of the outputs'
    buffers that do not belong to them stay as they were."""
    for k, o, lead in [(96, 64, 0), (96, 64, 3), (101, 67, 0), (64, 72, 8)]:
        big = rand(3, 50, lead + k + 5, seed=1, dtype=dtype).cuda()
        x = big[:, 4:41, lead:lead + k]
        wbig = rand(o + 2, lead + k + 3, seed=2, dtype=dtype, scale=0.1).cuda()
        w = wbig[1:o + 1, lead:lead + k]
        b = rand(o + 3, seed=3, dtype=dtype).cuda()[3:]
        res = rand(37, 3, o + 1, seed=4, dtype=dtype).cuda().transpose(0, 1)[..., 1:]
        gate = rand(3, 37, o + 7, seed=5, dtype=dtype).cuda()[..., 7:]
        buf = torch.full((37, 3, o + 9), 7.0, dtype=dtype, device="cuda")
        out = buf.transpose(0, 1)[..., 2:o + 2]
        y, pre = sv.linear(x, w, b, act="silu", gate=gate, residual=res, want_pre=True, out=out)
        assert y is out
        Y, Z, by, bz = linear64(x, w, b, "silu", gate, res)
        close(out, Y, by)
        assert bool((buf[..., :2] == 7).all()) and bool((buf[..., o + 2:] == 7).all())
        dy = rand(37, 3, o + 1, seed=6, dtype=dtype).cuda().transpose(0, 1)[..., :o]
        got = sv.linear_backward(dy, x, w, pre=pre, act="silu", gate=gate, want=["dx", "dw", "dbias", "dgate"])
        ref = linear_backward64(dy, x, w, pre, "silu", gate, UNIT[dtype])
        for name in got:
            close(got[name], *ref[name], name)
        got = sv.linear_backward(dy, x, w, want=["dx", "dw", "dbias"])  # dz is dy
        ref = linear_backward64(dy, x, w, None, unit=0.0)
        for name in got:
            close(got[name], *ref[name], name)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_residual_in_place_and_broadcast_inputs(dtype):
    x, w, b, g, r = inputs(dtype, 2, 90, 64, 136, True, "batch", True, seed=40)
    Y, _, by, _ = linear64(x, w, b, "none", g, r)
    y, _ = sv.linear(x, w, b, gate=g, residual=r, out=r)
    assert y is r
    close(r, Y, by)
    # one row of x for all tokens, one gate for the whole call
    one = x[:, :1].expand(2, 90, 64)
    gate = g[:1].expand(2, 136)
    y, pre = sv.linear(one, w, b, act="silu", gate=gate, want_pre=True)
    Y, _, by, _ = linear64(one, w, b, "silu", gate)
    close(y, Y, by)
    got = sv.linear_backward(y, one, w, pre=pre, act="silu", gate=gate, want=["dw", "dgate"])
    ref = linear_backward64(y, one, w, pre, "silu", gate, UNIT[dtype])
    close(got["dw"], *ref["dw"])
    close(got["dgate"], *ref["dgate"])


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_infinities_stay_in_their_rows(dtype):
    """A row with an infinity or NaN spoils its own outputs only: nothing of a tile's padding is multiplied into others."""
    for N, k, o in [(3, 70, 40), (150, 70, 40), (300, 96, 264)]:
        x, w, b, _, _ = inputs(dtype, 1, N, k, o, True, "none", False, seed=50)
        clean, _ = sv.linear(x, w, b)
        x[0, N - 1, k - 1] = float("inf")
        x[0, 1, 0] = float("nan")
        y, _ = sv.linear(x, w, b)
        keep = [n for n in range(N) if n not in (1, N - 1)]
        assert torch.equal(y[0, keep], clean[0, keep])
        assert bool(y[0, 1].isnan().all()) and not bool(y[0, N - 1].isfinite().any())
        dy = torch.ones_like(y)
        dx = sv.linear_backward(dy, x, w, want=["dx"])["dx"]
        assert bool(dx.isfinite().all())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_far_out(act):
    """Values and slopes of large arguments are the limits, without NaN."""
    z = torch.tensor([-3e38, -1e20, -1e10, -200.0, -30.0, -0.0, 0.0, 30.0, 200.0, 1e10, 1e20, 3e38], device="cuda")
    w = torch.ones(1, 1, device="cuda")
    y, pre = sv.linear(z[:, None], w, act=act, want_pre=True)
    assert torch.equal(pre[:, 0], z)
    want = torch.where(z > 0, z, torch.zeros_like(z))
    assert torch.allclose(y[:, 0], want, rtol=1e-6, atol=1e-11)  # 30 / e^30 is 3e-12
    d = sv.linear_backward(torch.ones_like(y), None, w, pre=pre, act=act, want=["dx"])["dx"][:, 0]
    slope = torch.where(z == 0, torch.full_like(z, 0.5), (z > 0).float())
    assert torch.allclose(d, slope, rtol=1e-6, atol=1e-10)


def test_results_do_not_depend_on_stream_or_workspace():
    """The same call on a side stream, among other work, gives the same bits."""
    x, w, b, g, r = inputs(torch.bfloat16, 2, 333, 520, 264, True, "token", True, seed=60)
    y0, _ = sv.linear(x, w, b, act="gelu", gate=g, residual=r)
    dy = rand(2, 333, 264, seed=61, dtype=torch.bfloat16).cuda()
    g0 = sv.linear_backward(dy, x, w, pre=y0, act="gelu", gate=g, want=["dx", "dw", "dbias", "dgate"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    junk = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    del junk  # the next workspace holds NaN patterns
    with torch.cuda.stream(side):
        y1, _ = sv.linear(x, w, b, act="gelu", gate=g, residual=r)
        g1 = sv.linear_backward(dy, x, w, pre=y0, act="gelu", gate=g, want=["dx", "dw", "dbias", "dgate"])
    y2, _ = sv.linear(x, w, b, act="gelu", gate=g, residual=r)
    torch.cuda.synchronize()
    assert torch.equal(y0, y1) and torch.equal(y0, y2)
    for name in g0:
        assert torch.equal(g0[name], g1[name]), name


def test_captured_and_replayed():
    """Forward and backward pass in one graph; every replay gives what the eager calls give on the same inputs."""
    x, w, b, g, r = inputs(torch.bfloat16, 2, 75, 264, 136, True, "batch", True, seed=70)
    dy = rand(2, 75, 136, seed=71, dtype=torch.bfloat16).cuda()
    xs, dys = torch.empty_like(x), torch.empty_like(dy)

    def step(x, dy):
        y, pre = sv.linear(x, w, b, act="silu", gate=g, residual=r, want_pre=True)
        return [y, *sv.linear_backward(dy, x, w, pre=pre, act="silu", gate=g, want=["dx", "dw", "dbias", "dgate"]).values()]

    xs.copy_(x), dys.copy_(dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(xs, dys)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(xs, dys)
    for k in range(3):
        x2, dy2 = rand(*x.shape, seed=80 + k, dtype=x.dtype).cuda(), rand(*dy.shape, seed=90 + k, dtype=x.dtype).cuda()
        xs.copy_(x2), dys.copy_(dy2)
        graph.replay()
        ref = step(x2, dy2)
        torch.cuda.synchronize()
        for a, e in zip(out, ref):
            assert torch.equal(a, e)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_rows_that_lie_more_than_4_gib_apart(dtype):
    """Element offsets past 32 bits in x, w, the gate, the residual and the output."""
    far = (1 << 31) + 72
    n, k, o = 3, 72, 40

    def rows(count, width, seed):
        buf = torch.empty(far * (count - 1) + width, dtype=dtype, device="cuda")
        t = buf.as_strided((count, width), (far, 1))
        t.copy_(rand(count, width, seed=seed, dtype=dtype))
        return t

    x, res, gate = rows(n, k, 1), rows(n, o, 2), rows(n, o, 3)
    w = rand(o, k, seed=4, dtype=dtype, scale=0.1).cuda()
    out = rows(n, o, 5)
    sv.linear(x, w, act="silu", gate=gate, residual=res, out=out)
    Y, _, by, _ = linear64(x, w, None, "silu", gate, res)
    close(out, Y, by)
    del res, out
    many = rand(70, k, seed=6, dtype=dtype).cuda()  # the tile kernel: the weights' rows far apart
    wf = rows(2, k, 7)
    y, _ = sv.linear(many, wf)
    Y, _, by, _ = linear64(many, wf)
    close(y, Y, by)
    got = sv.linear_backward(rand(n, o, seed=8, dtype=dtype).cuda(), x, w, want=["dx", "dw"])
    ref = linear_backward64(rand(n, o, seed=8, dtype=dtype), x, w, None, unit=0.0)
    for name in got:
        close(got[name], *ref[name], name)


def test_calls_on_two_streams_at_once():
    """Forward and backward passes of two sizes on two streams side by side give what they give alone."""
    a = inputs(torch.bfloat16, 2, 700, 1000, 520, True, "batch", True, seed=400)
    b = inputs(torch.bfloat16, 1, 900, 333, 1111, True, "token", True, seed=410)

    def step(x, w, bias, g, r):
        y, pre = sv.linear(x, w, bias, act="gelu_tanh", gate=g, residual=r, want_pre=True)
        return [y, *sv.linear_backward(y, x, w, pre=pre, act="gelu_tanh", gate=g, want=["dx", "dw", "dbias", "dgate"]).values()]

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


def test_captured_large_tiles():
    """The 256 x 256 tiles, whose LDS is all of a CU's, recorded and replayed."""
    x, w, b, _, r = inputs(torch.bfloat16, 1, 4100, 136, 4104, True, "none", True, seed=420)
    xs = x.clone()
    sv.linear(xs, w, b, residual=r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = sv.linear(xs, w, b, residual=r)
        dx = sv.linear_backward(y, xs, w, want=["dx"])["dx"]
    for k in range(3):
        x2 = rand(*x.shape, seed=430 + k, dtype=x.dtype).cuda()
        xs.copy_(x2)
        graph.replay()
        y2, _ = sv.linear(x2, w, b, residual=r)
        dx2 = sv.linear_backward(y2, x2, w, want=["dx"])["dx"]
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(dx, dx2)


# batches of one token each: their rows count as one entry's
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("gate", ["none", "batch", "token", "shared"])
@pytest.mark.parametrize("size", [(1, 1, 40, 24), (2, 1, 40, 24), (70, 1, 33, 67), (1300, 1, 64, 264)], ids=str)
def test_batches_of_one_token(size, gate, dtype):
    B, N, k, o = size
    x, w, b, g, _ = inputs(dtype, *size, bias=True, gate=gate if gate != "shared" else "none", residual=False, seed=7)
    if gate == "shared":
        g = rand(o, seed=8, dtype=dtype).cuda().expand(B, o)
    _, pre = sv.linear(x, w, b, act="gelu", gate=g, want_pre=True)
    big = rand(B, 3, o + 5, seed=9, dtype=dtype).cuda()
    dy = big[:, 1:2, 2:2 + o]
    want = ["dx", "dw", "dbias"] + (["dgate"] if g is not None else [])
    got = sv.linear_backward(dy, x, w, pre=pre, act="gelu", gate=g, want=want)
    ref = linear_backward64(dy, x, w, pre, "gelu", g, UNIT[dtype])
    for name in want:
        close(got[name], ref[name][0], ref[name][1], name)


def test_batches_past_the_longest_launch():
    """2^24 batch entries are as many workgroups of the gradient's kernel, 2^32 threads."""
    B = (1 << 24) + 5
    for N in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(N)
        dy = torch.randn(B, N, 8, device="cuda", generator=g).bfloat16()
        pre = torch.randn(B, N, 8, device="cuda", generator=g).bfloat16()
        gate = torch.randn(B, 8, device="cuda", generator=g).bfloat16()
        got = sv.linear_backward(dy, None, None, pre=pre, act="silu", gate=gate, want=["dgate"])["dgate"]
        for at in (0, B // 2, B - 300):
            part = slice(at, at + 300)
            ref = linear_backward64(dy[part], None, None, pre[part], "silu", gate[part], UNIT[torch.bfloat16])["dgate"]
            close(got[part], *ref, f"{N} {at}")


def test_the_most_rows():
    """2^30 rows, in more tiles than one launch may hold threads for along one axis. d_in = 1: the products are exact in fp32 and
    rounded once, as torch's are."""
    rows = 1 << 30
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(1 << 20, 1, device="cuda", generator=g).bfloat16().repeat(rows >> 20, 1)
    w = rand(1, 1, seed=4, dtype=torch.bfloat16).cuda()
    x[-5:] = 3.0
    y, _ = sv.linear(x, w)
    for at in range(0, rows, 1 << 27):
        part = slice(at, at + (1 << 27))
        assert torch.equal(y[part], x[part] * w)


# 9 to 256 rows, and one more, with weights whose rows lie at odd addresses: odd lengths, shorter than 16 bytes, longer than
# a step (32 fp32) by one, tiles of both kinds, a contraction in parts; as slices of a larger tensor at every offset
ODD_FEW = [(1, 9, 1003, 17000), (1, 64, 131, 259), (1, 65, 131, 259), (2, 32, 5001, 129), (1, 12, 4239, 5), (1, 10, 1, 1), (1, 20, 3, 17000),
           (1, 33, 33, 67), (4, 8, 65, 33), (1, 256, 131, 259), (1, 257, 131, 67), (2, 100, 1003, 17)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("lead", [0, 1, 2, 3])
@pytest.mark.parametrize("size", ODD_FEW, ids=str)
def test_few_rows_with_weights_at_odd_addresses(size, lead, dtype):
    i = ODD_FEW.index(size)
    x, w, b, g, r = inputs(dtype, *size, bias=True, gate="token", residual=True, seed=600 + i)
    o, k = w.shape
    big = torch.full((o, lead + k + 1 + lead), float("nan"), dtype=dtype, device="cuda")
    big[:, lead:lead + k] = w
    w = big[:, lead:lead + k]
    y, pre = sv.linear(x, w, b, act="silu", gate=g, residual=r, want_pre=True)
    Y, Z, by, bz = linear64(x, w, b, "silu", g, r)
    close(pre, Z, bz, "pre")
    close(y, Y, by, "y")
    dy = rand(*pre.shape, seed=700 + i, dtype=dtype).cuda()
    got = sv.linear_backward(dy, x, w, pre=pre, act="silu", gate=g, want=["dx", "dw", "dbias"])
    ref = linear_backward64(dy, x, w, pre, "silu", g, UNIT[dtype])
    for name in got:
        close(got[name], *ref[name], name)
