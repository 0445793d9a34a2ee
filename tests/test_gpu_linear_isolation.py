"""linear and its gradients: nothing of the workspace's former contents, of other rows and columns, or of values past the range of an
exponential reaches a result."""
import ctypes
import math

import pytest
import torch

import paper_2603_08982_amd as sv
from projection_helpers import UNIT, act64, f64
from test_gpu_linear import NAMES, TYPES, inputs, rand

pytestmark = pytest.mark.gpu
CODE = {torch.float32: 0, torch.bfloat16: 1}
ACT = {"none": 0, "silu": 1, "gelu": 2, "gelu_tanh": 3}


def two(t):
    return (ctypes.c_int64 * 2)(t.stride(0), t.stride(1))


def workspace(need, fill):
    """A workspace of exactly that size and alignment, between bytes that must stay as they are."""
    big = torch.full((need + 1024,), 0x5a, dtype=torch.uint8, device="cuda")
    at = -big.data_ptr() % 256 + 256
    big[at:at + need] = fill
    return big, at


def whole(big, at, need):
    assert bool((big[:at] == 0x5a).all()) and bool((big[at + need:] == 0x5a).all())


# odd lengths (copies of both operands, zeros behind the values of dz), contractions in parts (of the forward pass, dx and dw), few
# rows, an even one
SIZES = [(2, 37, 131, 67), (2, 150, 4103, 71), (1, 300, 72, 4101), (1, 4001, 33, 65), (3, 1, 131, 67), (2, 1, 5000, 72), (1, 64, 8200, 16), (2, 75, 104, 72)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_what_the_workspace_held_does_not_matter(size, dtype):
    """Filled with NaN patterns and with zeros, the same bits; and not a byte around it is written."""
    B, N, k, o = size
    lib, dt, act = sv.load_library(), CODE[dtype], ACT["silu"]
    big_x = rand(B, N + 1, k, seed=1, dtype=dtype).cuda()
    x = big_x[:, :N]  # batches apart
    w = rand(o, k, seed=2, dtype=dtype, scale=k ** -0.5).cuda()
    bias, gate = rand(o, seed=3, dtype=dtype).cuda(), rand(B, o, seed=4, dtype=dtype).cuda()
    dy = rand(B, N, o + 3, seed=5, dtype=dtype).cuda()[..., 1:o + 1]  # rows at odd addresses
    gst = (ctypes.c_int64 * 2)(o, 0)
    s = torch.cuda.current_stream().cuda_stream
    results = []
    for fill in (0xff, 0, 0x7f):
        y, pre = torch.full((2, B, N, o), float("nan"), dtype=dtype, device="cuda")
        need = lib.svgear_linear_workspace(x.data_ptr(), two(x), w.data_ptr(), k, dt, B, N, k, o)
        ws, at = workspace(need, fill)
        assert lib.svgear_linear(x.data_ptr(), two(x), w.data_ptr(), k, bias.data_ptr(), dt, B, N, k, o, act, gate.data_ptr(), gst, None, None,
                                 pre.data_ptr(), y.data_ptr(), two(y), ws.data_ptr() + at, need, s) == 0
        whole(ws, at, need)
        dx = torch.full((B, N, k), float("nan"), dtype=dtype, device="cuda")
        dw = torch.full((o, k), float("nan"), dtype=dtype, device="cuda")
        dbias, dgate = torch.full((o,), float("nan"), dtype=dtype, device="cuda"), torch.full((B, o), float("nan"), dtype=dtype, device="cuda")
        head = (dy.data_ptr(), two(dy), x.data_ptr(), two(x), w.data_ptr(), k)
        need = lib.svgear_linear_backward_workspace(*head, dt, B, N, k, o)
        ws, at = workspace(need, fill)
        assert lib.svgear_linear_backward(*head, pre.data_ptr(), dt, B, N, k, o, act, gate.data_ptr(), gst, dx.data_ptr(), two(dx), dw.data_ptr(),
                                          dbias.data_ptr(), dgate.data_ptr(), ws.data_ptr() + at, need, s) == 0
        whole(ws, at, need)
        results.append([y, pre, dx, dw, dbias, dgate])
    for got in results:
        for a, b in zip(results[0], got):
            assert bool(a.isfinite().all()) and torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("size", [(3, 70, 40), (12, 33, 67), (151, 70, 41), (301, 131, 265), (257, 64, 4101)], ids=str)
def test_gradients_of_other_rows_and_columns_stay_clean(size, act, dtype):
    """An infinity or NaN of dy spoils its row of dx and its column's row of dw and dbias, one of x its column of dw; what is behind the
    last row, column or element of a contraction, or repeats the last, reaches no other."""
    N, k, o = size
    x, w, b, _, _ = inputs(dtype, 1, N, k, o, True, "none", False, seed=50)
    _, pre = sv.linear(x, w, b, act=act, want_pre=True)
    dy = rand(1, N, o, seed=51, dtype=dtype).cuda()
    back = lambda dy, x: sv.linear_backward(dy, x, w, pre=pre, act=act, want=["dx", "dw", "dbias"])
    clean = back(dy, x)
    bad_dy, bad_x = dy.clone(), x.clone()
    bad_dy[0, N - 1, o - 1] = float("inf")
    bad_dy[0, 1, 0] = float("nan")
    bad_x[0, N - 1, k - 1] = float("nan")
    bad_x[0, 0, 3] = float("-inf")
    got = back(bad_dy, bad_x)
    rows = [n for n in range(N) if n not in (1, N - 1)]
    assert torch.equal(got["dx"][0, rows], clean["dx"][0, rows])
    assert bool(got["dx"][0, 1].isnan().all()) and not bool(got["dx"][0, N - 1].isfinite().any())
    outs, ins = list(range(1, o - 1)), [i for i in range(k) if i not in (3, k - 1)]
    assert torch.equal(got["dw"][outs][:, ins], clean["dw"][outs][:, ins])
    for at in (got["dw"][0], got["dw"][o - 1], got["dw"][:, 3], got["dw"][:, k - 1]):
        assert not bool(at.isfinite().any())
    assert torch.equal(got["dbias"][outs], clean["dbias"][outs]) and not bool(got["dbias"][[0, o - 1]].isfinite().any())


FAR = [-3e38, -1e20, -1e10, -200.0, -90.0, -88.5, -30.0, -10.0, -4.0, -0.0, 0.0, 4.0, 10.0, 30.0, 88.5, 90.0, 200.0, 1e10, 1e20, 3e38]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("rows, width", [(3, 40), (20, 24), (20, 21), (300, 72)])
def test_activations_and_slopes_far_out(rows, width, act, dtype):
    """Through weights that are the unit matrix, so that y = act(x) and dx = act'(x), in the epilogues of few rows, of eight columns and of
    single ones. An argument of an exponential up to 2^7, found in four operations, puts 2^9 half steps on it, the hardware's own
    2^-17: 2^-14 in all. An exponential past fp32 makes the rest, below 89 / 2^128, zero."""
    z = torch.tensor([FAR[(i + 3 * r) % len(FAR)] for r in range(rows) for i in range(width)]).view(rows, width).to(dtype).cuda()
    eye = torch.eye(width, dtype=dtype, device="cuda")
    y, pre = sv.linear(z, eye, act=act, want_pre=True)
    assert torch.equal(pre, z)
    dx = sv.linear_backward(torch.ones_like(y), None, eye, pre=pre, act=act, want=["dx"])["dx"]
    Z = f64(z)
    near = Z.clamp(-1e6, 1e6).requires_grad_(True)  # beyond, the limits
    value = act64(near, act) if act == "gelu" else near * torch.sigmoid(near if act == "silu" else (8 / math.pi) ** 0.5 * (near + 0.044715 * near ** 3))
    slope, = torch.autograd.grad(value.sum(), near)
    want = torch.where(Z.abs() > 1e6, Z.clamp(min=0.0), value.detach())
    for got, ref in ((y, want), (dx, slope)):
        off = (f64(got) - ref).abs() - ((UNIT[dtype] + 2.0 ** -14) * ref.abs() + 2.0 ** -121)
        assert bool((off <= 0).all()), (float(Z.flatten()[off.argmax()]), float(f64(got).flatten()[off.argmax()]), float(ref.flatten()[off.argmax()]))
