"""svgear_rotary and its backward pass with norms, over the whole range of values that they take."""
import pytest
import torch

import paper_2603_08982_amd as sv
from projection_helpers import close, rotary64, rotary_backward64
from test_gpu_rotary import NAMES, TYPES, rand, setup

pytestmark = pytest.mark.gpu

# one wave a token and several, heads of both sizes, text tokens
SHAPES = [(2, 5, (2, 3, 4), 0, 3, 64, (10, 11, 11)), (1, 40, (1, 3, 4), 0, 2, 128, (22, 21, 21))]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("scale, eps", [(1e13, 1e-6), (1e15, 1e-6), (1e16, 1e-6), (1e16, 0.0), (1e-4, 1e-6), (1e-13, 0.0), (1e-15, 0.0),
                                        (1e-15, 1e-30), (1e-17, 0.0)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norms_of_large_and_small_values(shape, scale, eps, halves, norm, dtype):
    """x of rms 1.5 times `scale`: up to 1e17, and, without an eps that hides it, down to where squares are still normal numbers."""
    q, k, f, sections, weights, kw = setup(shape, dtype, norm, None, seed=11)
    kw["eps"] = eps
    q, k = ((t.float() * scale).to(dtype) for t in (q, k))
    assert float(max(q.abs().max(), k.abs().max())) <= 1e17
    out = sv.rotary([q, k], f, sections, weights=weights, halves=halves, **kw)
    grads = [rand(*q.shape, seed=12 + t, dtype=dtype).cuda() for t in range(2)]
    dx, dweight = sv.rotary_backward(grads, [q, k], f, sections, weights=weights, halves=halves, **kw)
    for t, x in enumerate((q, k)):
        close(out[t], *rotary64(x, f, sections, weight=weights[t], halves=halves, **kw), "y")
        rdx, bdx, rdw, bdw = rotary_backward64(grads[t], x, f, sections, weight=weights[t], halves=halves, **kw)
        close(dx[t], rdx, bdx, "dx")
        close(dweight[t], rdw, bdw, "dweight")


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("eps", [1e-6, 1e-20, 1e-30, 1e-37])
def test_gradient_of_rows_of_zeros(eps, norm, dtype):
    """Zeros are as the smallest values: dx = g / sqrt(eps), which is finite for every eps but 0, and nothing comes to dweight."""
    q, k, f, sections, weights, kw = setup(SHAPES[0], dtype, norm, None, seed=21)
    kw["eps"] = eps
    q[:, :, 3] = 0.0
    q[1, :, 25] = 0.0
    g = rand(*q.shape, seed=22, dtype=dtype).cuda()
    (dx,), (dw,) = sv.rotary_backward([g], [q], f, sections, weights=weights[:1], **kw)
    rdx, bdx, rdw, bdw = rotary_backward64(g, q, f, sections, weight=weights[0], **kw)
    assert bool(dx.isfinite().all())
    close(dx, rdx, bdx, "dx")
    close(dw, rdw, bdw, "dweight")


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("scale, dy_scale, eps", [(1e16, 1e16, 1e-6), (1e16, 1e-16, 1e-6), (1.0, 1e16, 1e-6), (1.0, 1e-20, 1e-6),
                                                  (1e-15, 1e16, 0.0), (1e-15, 1e-15, 0.0)])
def test_gradients_of_any_size(scale, dy_scale, eps, norm, dtype):
    q, _, f, sections, weights, kw = setup(SHAPES[1], dtype, norm, None, seed=31)
    kw["eps"] = eps
    q = (q.float() * scale).to(dtype)
    g = (rand(*q.shape, seed=32) * dy_scale).to(dtype).cuda()
    (dx,), (dw,) = sv.rotary_backward([g], [q], f, sections, weights=weights[:1], **kw)
    rdx, bdx, rdw, bdw = rotary_backward64(g, q, f, sections, weight=weights[0], **kw)
    close(dx, rdx, bdx, "dx")
    close(dw, rdw, bdw, "dweight")
