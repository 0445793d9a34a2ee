"""The layer norm and its gradients against plain 64-bit forms."""
import pytest
import torch

import paper_2603_08982_amd as sv
from dense_helpers import close, norm64, norm_backward64

pytestmark = pytest.mark.gpu

EPS = 1e-6


def make(seed, dtype, B, N, c, affine, mod, far=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = lambda *s, scale=1.0, mean=0.0: (torch.randn(*s, generator=g, device="cuda") * scale + mean).to(dtype)
    x = t(B, N, c, mean=far)
    w, b = (t(c, scale=0.2, mean=1.0), t(c, scale=0.3)) if affine else (None, None)
    shape = {"none": None, "batch": (B, c), "token": (B, N, c)}[mod]
    s, h = (t(*shape, scale=0.3), t(*shape, scale=0.3)) if shape else (None, None)
    return x, w, b, s, h, t(B, N, c)


# (lanes of one row: 8, 16, 32, 64; runs of eight columns a lane: 1, 2, 4; waves a row: 1 to 16; odd lengths of each)
WIDTHS = [1, 7, 8, 48, 65, 100, 129, 255, 256, 257, 512, 513, 1003, 1541, 2048, 5120, 8191, 8200, 12288, 16384, 16391, 20480, 32768]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("c", WIDTHS)
def test_widths(c, dtype):
    for B, N, affine, mod in ((2, 5, True, "batch"), (1, 9, False, "none"), (2, 3, True, "token"), (3, 1, False, "batch")):
        x, w, b, s, h, dy = make(c, dtype, B, N, c, affine, mod)
        y = sv.layer_norm(x, w, b, scale=s, shift=h, eps=EPS)
        want, e, *_ = norm64(x, w, b, s, h, EPS)
        close(y, want, e, (B, N, c, mod))
        names = ["dx"] + (["dweight", "dbias"] if affine else []) + (["dscale", "dshift"] if mod != "none" else [])
        got = sv.layer_norm_backward(dy, x, w, b, scale=s, eps=EPS, want=names)
        ref = norm_backward64(dy, x, w, b, s, EPS)
        for n in names:
            close(got[n], ref[n][0], ref[n][1], (n, B, N, c, mod))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,N,c,mod", [(1, 3001, 48, "none"), (3, 2111, 96, "batch"), (2, 1500, 513, "token"), (1, 4999, 640, "batch"),
                                       (40, 17, 1024, "batch"), (500, 2, 72, "batch"), (1, 1, 5120, "batch"), (2, 2100, 5120, "batch")])
def test_many_rows(B, N, c, mod, dtype):
    x, w, b, s, h, dy = make(B + N + c, dtype, B, N, c, True, mod)
    close(sv.layer_norm(x, w, b, scale=s, shift=h, eps=EPS), *norm64(x, w, b, s, h, EPS)[:2], "y")
    names = ["dx", "dweight", "dbias"] + (["dscale", "dshift"] if mod != "none" else [])
    got = sv.layer_norm_backward(dy, x, w, b, scale=s, eps=EPS, want=names)
    ref = norm_backward64(dy, x, w, b, s, EPS)
    for n in names:
        close(got[n], *ref[n], n)


@pytest.mark.parametrize("far", [1e3, -3e4])
def test_rows_far_from_zero_keep_their_variance(far):
    x, w, b, s, h, dy = make(5, torch.float32, 2, 31, 1600, True, "batch", far)
    close(sv.layer_norm(x, w, b, scale=s, shift=h, eps=EPS), *norm64(x, w, b, s, h, EPS)[:2], "y")
    got = sv.layer_norm_backward(dy, x, w, b, scale=s, eps=EPS, want=["dx", "dweight"])
    ref = norm_backward64(dy, x, w, b, s, EPS)
    for n in got:
        close(got[n], *ref[n], n)


def test_one_value_far_from_the_others():
    x = torch.randn(6, 5120, device="cuda")
    x[:, 0], x[:, 4097] = 3e4, -2e4
    close(sv.layer_norm(x, eps=EPS), *norm64(x, None, None, None, None, EPS)[:2], "y")


def test_parts_of_weight_and_modulation():
    """weight, bias, scale and shift each alone."""
    x, w, b, s, h, dy = make(3, torch.bfloat16, 2, 19, 200, True, "batch")
    for kw in ({"weight": w}, {"bias": b}, {"scale": s}, {"shift": h}, {"weight": w, "shift": h}, {"bias": b, "scale": s}):
        full = {"weight": None, "bias": None, "scale": None, "shift": None, **kw}
        close(sv.layer_norm(x, **kw), *norm64(x, full["weight"], full["bias"], full["scale"], full["shift"], EPS)[:2], str(list(kw)))
    for want in (["dx"], ["dbias"], ["dweight"], ["dscale"], ["dshift"], ["dshift", "dx"], ["dweight", "dscale"]):
        got = sv.layer_norm_backward(dy, x, w, b, scale=s, want=want)
        ref = norm_backward64(dy, x, w, b, s, EPS)
        assert list(got) == want
        for n in want:
            close(got[n], *ref[n], n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_strides_and_alignment(dtype):
    B, N, c = 2, 23, 333
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)
    x, dy = r(N, B, c + 5)[:, :, 3:3 + c].transpose(0, 1), r(B, N + 2, c + 1)[:, 1:-1, 1:]
    mod = r(B, 6, c)  # the six vectors of a modulation
    s, h = mod[:, 1], mod[:, 4]
    buf = torch.full((B, N, c + 3), 7.0, device="cuda", dtype=dtype)
    y = sv.layer_norm(x, scale=s, shift=h, out=buf[:, :, 1:1 + c])
    close(y, *norm64(x, None, None, s, h, EPS)[:2], "y")
    assert (buf[:, :, 0] == 7).all() and (buf[:, :, 1 + c:] == 7).all()
    got = sv.layer_norm_backward(dy, x, scale=s, want=["dx", "dscale", "dshift"])
    ref = norm_backward64(dy, x, None, None, s, EPS)
    for n in got:
        close(got[n], *ref[n], n)
    st = r(N, c)  # a token's modulation, shared by the batch
    sh = st[None].expand(B, N, c)
    close(sv.layer_norm(x, scale=sh), *norm64(x, None, None, sh, None, EPS)[:2], "shared")
    one = r(1, c).expand(B, c)
    got = sv.layer_norm_backward(dy, x, scale=one, want=["dscale"])
    close(got["dscale"], *norm_backward64(dy, x, None, None, one, EPS)["dscale"], "one scale of all")
    two = sv.layer_norm(x[0], scale=s[0], shift=h[0])
    assert torch.equal(two, y[0])


def test_in_place():
    x, w, b, s, h, dy = make(4, torch.bfloat16, 2, 777, 640, True, "batch")
    y = sv.layer_norm(x, w, b, scale=s, shift=h)
    z = x.clone()
    assert sv.layer_norm(z, w, b, scale=s, shift=h, out=z) is z
    assert torch.equal(z, y)


def test_rows_do_not_meet():
    """A row of NaN or infinities spoils itself alone; the same rows elsewhere give the same bits."""
    x, w, b, *_ = make(6, torch.bfloat16, 1, 257, 776, True, "none")
    y = sv.layer_norm(x, w, b)
    z = x.clone()
    z[0, 100], z[0, 3, 5] = float("nan"), float("inf")
    u = sv.layer_norm(z, w, b)
    keep = [i for i in range(257) if i not in (3, 100)]
    assert torch.equal(u[0, keep], y[0, keep]) and u[0, 100].isnan().all()
    assert torch.equal(sv.layer_norm(x[:, 50:], w, b), y[:, 50:])


def test_gradient_against_differences():
    torch.manual_seed(0)
    x, w, b, s, h, dy = make(9, torch.float32, 2, 4, 40, True, "batch")
    got = sv.layer_norm_backward(dy, x, w, b, scale=s, want=["dx", "dweight", "dbias", "dscale", "dshift"])
    args = {"dx": x, "dweight": w, "dbias": b, "dscale": s, "dshift": h}
    for n, t in args.items():
        u = torch.randn_like(t)
        step = 2.0 ** -10
        f = lambda sign: norm64(*[(a.double() + sign * step * u.double()) if a is t else a.double() for a in (x, w, b, s, h)], EPS)[0]
        want = ((f(1) - f(-1)) * dy.double()).sum() / (2 * step)
        have = (got[n].double() * u.double()).sum()
        # third derivatives of order 1 over 6 times the step squared, summed over the gradients; fp32 on top
        room = (step ** 2 * 10 + 1e-5) * dy.abs().sum().double()
        assert abs(have - want) <= room, (n, have, want)


def test_captured():
    x, w, b, s, h, dy = make(2, torch.bfloat16, 2, 300, 1000, True, "batch")
    names = ["dx", "dweight", "dbias", "dscale", "dshift"]

    def both():
        return sv.layer_norm(x, w, b, scale=s, shift=h), sv.layer_norm_backward(dy, x, w, b, scale=s, want=names)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, r = both()
    for k in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        eager, grads = both()
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
        for n in names:
            assert torch.equal(r[n], grads[n]), (k, n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mod", ["batch", "token"])
@pytest.mark.parametrize("B,N,c", [(2, 19, 200), (3, 1, 65), (1, 777, 1003)])
def test_gradient_of_a_shift_alone(B, N, c, mod, dtype):
    """Without a scale (1 + scale) is 1, and dshift has the shift's shape."""
    x, w, b, s, h, dy = make(12, dtype, B, N, c, True, mod)
    ref = norm_backward64(dy, x, w, b, torch.zeros_like(s), EPS)
    for names in (["dshift"], ["dx", "dweight", "dbias", "dshift"]):
        got = sv.layer_norm_backward(dy, x, w, b, shift=h, want=names)
        assert got["dshift"].shape == h.shape
        for n in names:
            close(got[n], *ref[n], (n, B, N, c, mod))
    both, one = (sv.layer_norm_backward(dy, x, w, b, scale=s, want=["dx", "dscale", "dshift"], **kw) for kw in ({"shift": h}, {}))
    assert all(torch.equal(both[n], one[n]) for n in one)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,N,c", [(4, 3, 40), (5, 3, 40), (9, 130, 513), (300, 2, 5120), (2500, 3, 24), (20000, 2, 8)])
def test_many_entries(B, N, c, dtype):
    """Sums of a batch entry and of all of them: few entries by one workgroup, many dealt out and joined."""
    x, w, b, s, h, dy = make(B + c, dtype, B, N, c, True, "batch")
    names = ["dx", "dweight", "dbias", "dscale", "dshift"]
    got = sv.layer_norm_backward(dy, x, w, b, scale=s, eps=EPS, want=names)
    ref = norm_backward64(dy, x, w, b, s, EPS)
    for n in names:
        close(got[n], *ref[n], (n, B, N, c))
    for some in (["dscale", "dshift"], ["dweight"], ["dbias", "dscale"]):
        part = sv.layer_norm_backward(dy, x, w, b, scale=s, eps=EPS, want=some)
        assert all(torch.equal(part[n], got[n]) for n in some)


def test_entries_by_the_hundred_thousand():
    """As many batch entries as tokens of one: a second's work for one workgroup after the other, a millisecond's for all."""
    B, N, c = 600000, 2, 8
    x, w, b, s, h, dy = make(17, torch.float32, B, N, c, True, "batch")
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    sv.layer_norm_backward(dy, x, w, b, scale=s, want=["dscale"])
    begin.record()
    got = sv.layer_norm_backward(dy, x, w, b, scale=s, want=["dscale", "dshift", "dweight"])
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) < 200
    ref = norm_backward64(dy, x, w, b, s, EPS)
    for n in ("dscale", "dshift"):
        close(got[n], *ref[n], n)
    # (2^11 workgroups of 293 entries each, 32 of them one behind the other: 400 roundings as elsewhere)
    close(got["dweight"], *ref["dweight"], "dweight")
