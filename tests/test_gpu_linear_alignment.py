"""Results of linear and its gradients are functions of sizes, type and values: not of where the operands lie."""
import pytest
import torch

import paper_2603_08982_amd as sv
from test_gpu_linear import NAMES, TYPES, inputs, rand

pytestmark = pytest.mark.gpu


def moved(t, lead):
    """The same values in rows `lead` elements into longer ones."""
    big = torch.full((*t.shape[:-1], t.shape[-1] + lead + 5), float("nan"), dtype=t.dtype, device=t.device)
    big[..., lead:lead + t.shape[-1]] = t
    return big[..., lead:lead + t.shape[-1]]


# (rows, d_in, d_out): one part and several of the contraction, of the forward pass and of dx; more parts where tiles of 128 serve aligned
# rows than tiles of 64 would have (200 rows: 3 and 4, 100: 8 and 2); few rows, and more than are copied by the element
SIZES = [(1, 640, 200), (3, 1024, 96), (9, 1024, 264), (40, 4096, 512), (60, 520, 4104), (100, 20480, 8192), (200, 8192, 5120), (256, 5120, 8200),
         (257, 2048, 512), (700, 1024, 640)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_bits_do_not_depend_on_alignment(size, dtype):
    rows, k, o = size
    x, w, b, g, r = inputs(dtype, 0, rows, k, o, True, "token", True, seed=rows)
    dy = rand(rows, o, seed=rows + 9, dtype=dtype).cuda()

    def calls(place):
        y, pre = sv.linear(place(x), place(w), b, act="silu", gate=place(g), residual=place(r), want_pre=True)
        grads = sv.linear_backward(place(dy), place(x), place(w), pre=pre, act="silu", gate=place(g), want=["dx", "dw", "dbias", "dgate"])
        plain = sv.linear_backward(place(dy), place(x), place(w), want=["dx", "dw"])
        return {"y": y, "pre": pre, **grads, **{"plain " + n: t for n, t in plain.items()}}

    aligned = calls(lambda t: t)
    for lead in (1, 2, 3):
        got = calls(lambda t: moved(t, lead))
        for name in aligned:
            assert torch.equal(aligned[name], got[name]), (name, lead)
    only_w = sv.linear(x, moved(w, 1), b, act="silu", gate=g, residual=r)[0]
    assert torch.equal(aligned["y"], only_w)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("size", [(2, 2, 64, 40), (3, 1, 72, 136), (2, 100, 136, 72), (2, 300, 131, 67)], ids=str)
def test_bits_do_not_depend_on_strides(size, dtype):
    """Batches within tokens, tokens and batches far apart, and one row (stride 0) for a whole batch entry or call."""
    B, N, k, o = size
    x, w, b, g, r = inputs(dtype, B, N, k, o, True, "token", True, seed=B * N)
    dy = rand(B, N, o, seed=9, dtype=dtype).cuda()

    def far(t):
        big = torch.full((t.shape[0], t.shape[1], (1 << 21) + 8), float("nan"), dtype=t.dtype, device="cuda")
        big[..., :t.shape[2]] = t
        return big[..., :t.shape[2]]

    def calls(x, g, r, dy):
        y, pre = sv.linear(x, w, b, act="silu", gate=g, residual=r, want_pre=True)
        grads = sv.linear_backward(dy, x, w, pre=pre, act="silu", gate=g, want=["dx", "dw", "dbias"] + (["dgate"] if g.stride(1) else []))
        plain = sv.linear_backward(dy, x, w, want=["dx", "dw"])
        return {"y": y, "pre": pre, **grads, **{"plain " + n: t for n, t in plain.items()}}

    inner = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    one_of_each = lambda t: t[:, :1].expand(-1, N, -1)
    one = lambda t: t[:1, :1].expand(B, N, -1)
    for place in (inner, far, one_of_each, one):
        args = [place(t) for t in (x, g, r, dy)]
        want, got = calls(*[t.contiguous() for t in args]), calls(*args)
        for name in got:
            assert torch.equal(want[name], got[name]), name
