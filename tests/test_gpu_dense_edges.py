"""Dense attention and its gradients at the far ends of what they take, against plain 64-bit forms."""
import pytest
import torch

import paper_2603_08982_amd as sv
from dense_helpers import attention64, attention_backward64, close
from test_gpu_dense_attention import BF, F, check, make, slopes_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_distances_behind_a_long_past(causal, dtype, d):
    """Positions that fp32 has no numbers for: 37 queries at the end of 2^25 + 77 keys, of which all but the last 512 are zeros and
    weigh e^-59 at most, that is 2^25 times 1e-26 beside a sum of 0.01 at least."""
    near, n = 512, (1 << 25) + 77
    q, k, v, dy = make(41, dtype, 1, 2, 1, 37, near, d)
    slopes = torch.tensor([0.5, 0.125], device="cuda")
    far_k, far_v = (torch.zeros(1, 1, n, d, dtype=dtype, device="cuda") for _ in range(2))
    far_k[:, :, -near:], far_v[:, :, -near:] = k, v
    kw = {"causal": causal, "slopes": slopes}
    o, lse = sv.attention(q, far_k, far_v, want_lse=True, **kw)
    want, e, want_lse, el = attention64(q, k, v, **kw)
    close(lse, want_lse, el, "lse")
    close(o, want, e, "o")
    got = sv.attention_backward(dy, q, far_k, far_v, o, lse, **kw)
    ref = attention_backward64(dy, q, k, v, o, lse, **kw)
    close(got["dq"], *ref["dq"], "dq")
    for name in ("dk", "dv"):
        close(got[name][:, :, -near:], *ref[name], name)
        assert not got[name][:, :, :1 << 20].any(), name
    del far_k, far_v, got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64), (F, 128)])
@pytest.mark.parametrize("Nq,Nk", [(37, 5003), (1500, 70)])
def test_distances_over_many_parts(Nq, Nk, dtype, d):
    q, k, v, dy = make(42, dtype, 1, 6, 3, Nq, Nk, d)
    for kw in ({}, {"causal": True, "cap": 20.0}):
        check(q, k, v, dy, (Nq, Nk, kw), slopes=slopes_of(6), **kw)
