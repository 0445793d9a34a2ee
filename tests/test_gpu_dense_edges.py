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


def relative_scores(monkeypatch):
    """scores64 with a bound that is relative to the score, for any cap. In half steps (U32): the series for small scores is the best fit of its
    degree to 10 (bf16) or below 1 (fp32), its coefficients' factors 4, its sums 4; the exponential and reciprocal some 10, see
    the factors below; the cap's product and the sum 2."""
    import dense_helpers

    plain = dense_helpers.scores64

    def scores(q, k, scale, cap, slopes, **mask):
        s, e, keeps, seen = plain(q, k, scale, None, slopes, **mask)
        if cap:
            full, _, keeps, _ = plain(q, k, scale, cap, slopes, **mask)
            raw = plain(q, k, scale, cap, None, **mask)[0]
            # what the product is off by counts by the slope, which is 1 at most
            e = e + torch.where(seen, 24 * dense_helpers.U32 * raw.abs(), 0.0)
            if q.dtype == BF and cap <= 256:
                e = e + torch.where(seen, 16 * dense_helpers.U32 * cap, 0.0)
            s = full
        return s, e, keeps, seen

    monkeypatch.setattr(dense_helpers, "scores64", scores)


# (cap, scale or none: with one of 8 scores are of the size of a cap of some hundreds)
CAPS = [(256.0, None), (256.0, 8.0), (257.0, 8.0), (1000.0, 8.0), (1e3, None), (3e4, None), (1e6, None), (1e6, -0.125), (1e9, None)]


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64), (F, 128)])
@pytest.mark.parametrize("kw", [{}, {"causal": True}, {"slopes": True}, {"slopes": True, "causal": True}], ids=str)
@pytest.mark.parametrize("cap,scale", CAPS)
def test_large_caps(monkeypatch, cap, scale, kw, dtype, d):
    """Far from its cap a score is what it was, whatever the cap; 203 keys are no whole tiles."""
    relative_scores(monkeypatch)
    q, k, v, dy = make(43, dtype, 1, 4, 2, 140, 203, d, spread=2.0)
    kw = dict(kw, slopes=slopes_of(4)) if "slopes" in kw else kw
    check(q, k, v, dy, (cap, scale, kw), cap=cap, scale=scale, **kw)


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_cap_out_of_reach_is_none(dtype):
    """Scores of some units under a cap of 2^40 are those without one, to their last digits, in both passes."""
    q, k, v, dy = make(44, dtype, 2, 4, 4, 130, 333, 64)
    plain, far = check(q, k, v, dy, "without"), sv.attention(q, k, v, want_lse=True, cap=2.0 ** 40)
    # bf16: weights and results of both are rounded once, 4 times 2^-8; fp32: 24 half steps of scores up to 8
    tol = 2.0 ** -6 if dtype == BF else 24 * 2.0 ** -24 * 8
    assert (far[0].double() - plain[0].double()).norm() <= tol * plain[0].double().norm()
    got = sv.attention_backward(dy, q, k, v, *far, cap=2.0 ** 40)
    for n in got:
        assert (got[n].double() - plain[2][n].double()).norm() <= 2 * tol * plain[2][n].double().norm(), n


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64), (F, 128)])
@pytest.mark.parametrize("kw", [{}, {"causal": True}, {"slopes": True, "cap": 300.0}, {"docs": True}], ids=str)
@pytest.mark.parametrize("Nq,Nk", [(64, 64), (70, 70), (33, 97), (1, 1), (5, 2003), (700, 65), (130, 191), (1, 999)])
def test_an_infinity_in_the_last_row(Nq, Nk, kw, dtype, d):
    """What the last key's value has, and in the gradients the last query's dy, comes out as the formula says, whether or not the rows are
    whole tiles: an infinity in a column is one of the rows that see it, and touches no other column."""
    q, k, v, dy = make(45, dtype, 2, 4, 2, Nq, Nk, d, spread=0.5)
    kw = dict(kw)
    if "slopes" in kw:  # (so flat that no weight vanishes)
        kw["slopes"] = torch.full((4,), 1e-3, device="cuda")
    if kw.pop("docs", False):  # a document in front, a document of the rest, one row of padding
        if Nq < 4:
            return
        kw.update(q_offsets=torch.tensor([0, 2, Nq - 1], dtype=torch.int32, device="cuda"),
                  k_offsets=torch.tensor([0, 3, Nk - 1], dtype=torch.int32, device="cuda"))
    last_q, last_k = (int(kw[n][-1]) if n in kw else e for n, e in (("q_offsets", Nq), ("k_offsets", Nk)))
    what = (Nq, Nk, list(kw), dtype, d)
    plain = [t.clone() for t in (v, dy)]
    v[:, :, last_k - 1, 3], v[:, :, last_k - 1, d - 1] = float("inf"), -float("inf")
    o, lse = sv.attention(q, k, v, want_lse=True, **kw)
    want, e, want_lse, el = attention64(q, k, plain[0], **kw)
    close(lse, want_lse, el, ("lse", what))
    mid = torch.arange(d, device="cuda")
    mid = mid[(mid != 3) & (mid != d - 1)]
    close(o[..., mid], want[..., mid], e[..., mid], ("o", what))
    first = 2 if "q_offsets" in kw else 0
    sees = torch.arange(Nq, device="cuda") >= (last_q - 1 if kw.get("causal") else first)
    sees &= torch.arange(Nq, device="cuda") < last_q
    assert (o[:, :, sees, 3] == torch.inf).all() and (o[:, :, sees, d - 1] == -torch.inf).all(), what
    close(o[:, :, ~sees], want[:, :, ~sees], e[:, :, ~sees], ("o of others", what))

    o, lse = sv.attention(q, k, plain[0], want_lse=True, **kw)
    dy[:, :, last_q - 1, 3] = float("inf")
    got = sv.attention_backward(dy, q, k, plain[0], o, lse, **kw)["dv"]
    want, e = attention_backward64(plain[1], q, k, plain[0], o, lse, **kw)["dv"]
    others = torch.arange(d, device="cuda") != 3
    close(got[..., others], want[..., others], e[..., others], ("dv", what))
    seen = torch.arange(Nk, device="cuda") >= (3 if "k_offsets" in kw else 0)
    seen &= torch.arange(Nk, device="cuda") < last_k
    assert (got[:, :, seen, 3] == torch.inf).all(), what
    close(got[:, :, ~seen], want[:, :, ~seen], e[:, :, ~seen], ("dv of others", what))


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64), (F, 128)])
@pytest.mark.parametrize("cap", [1e37, 1e30, 1e-3, 1e-9, 1e-20, 1e-37])
def test_caps_at_the_ends_of_fp32(monkeypatch, cap, dtype, d):
    """Products are whole numbers, so that none is off by more than a small cap, and those of some tiles are all 0."""
    relative_scores(monkeypatch)
    g = torch.Generator(device="cuda")
    g.manual_seed(46)
    whole = lambda h, n: torch.randint(-2, 3, (2, h, n, d), generator=g, device="cuda").to(dtype)
    q, k = whole(4, 150), whole(2, 260)
    q[:, :, 40:80], k[:, :, 64:128] = 0, 0
    _, _, v, dy = make(46, dtype, 2, 4, 2, 150, 260, d)
    for kw in ({}, {"causal": True}, {"slopes": torch.full((4,), 0.01, device="cuda")}):
        check(q, k, v, dy, (cap, list(kw)), cap=cap, scale=0.125, **kw)


@pytest.mark.parametrize("dtype", [BF, F])
def test_more_heads_than_24_bits(dtype):
    """2^24 + 64 heads share a key head; their rows overlap, eight columns apart, and only the last 80 of dy are not 0."""
    H, n, d = (1 << 24) + 64, 80, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(47)

    def rows():
        flat = torch.zeros(8 * H + d, dtype=dtype, device="cuda")
        flat[8 * (H - n) + d - 8:] = torch.randn(8 * n + 8, generator=g, device="cuda").to(dtype)
        return flat.as_strided((1, H, 1, d), (0, 8, 0, 1))

    q, dy = rows(), rows()
    k, v = (torch.randn(1, 1, 2, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    o, lse = sv.attention(q, k, v, want_lse=True)
    got = sv.attention_backward(dy, q, k, v, o, lse, want=["dk", "dv"])
    last = [t[:, -n:].contiguous() for t in (dy, q)]
    ref = attention_backward64(last[0], last[1], k, v, o[:, -n:], lse[:, -n:])
    for name in got:
        close(got[name], *ref[name], name)
    del q, dy, o, lse
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F, 128), (F, 64)])
@pytest.mark.parametrize("row", [0, 1, 777, 2899])
def test_unbounded_rows_that_keys_behind_a_prefix_do_not_see(row, dtype, d):
    """3,000 queries over 100 keys, 10 of them a prefix: the first tile of keys reads all queries, and its keys from 10 on see the last 90 at
    most. A NaN in any query before those reaches the prefix alone. (Where such rows' elements are more than 2^31, the same takes minutes.)"""
    q, k, v, dy = make(48, dtype, 1, 2, 1, 3000, 100, d)
    kw = {"causal": True, "prefix": torch.tensor([10], dtype=torch.int32, device="cuda")}
    o, lse = sv.attention(q, k, v, want_lse=True, **kw)
    ref = attention_backward64(dy, q, k, v, o, lse, **kw)
    for spoilt in ("dy", "q"):
        Q, Y = q.clone(), dy.clone()
        (Y if spoilt == "dy" else Q)[:, :, row] = float("nan")
        got = sv.attention_backward(Y, Q, k, v, o, lse, **kw)
        for name in ("dk", "dv"):
            close(got[name][:, :, 10:], ref[name][0][:, :, 10:], ref[name][1][:, :, 10:], (name, spoilt))
            assert got[name][:, :, :10].isnan().all(), (name, spoilt)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64)])
@pytest.mark.parametrize("docs", [62, 63, 64, 65, 127, 1000, 4097])
def test_many_documents(docs, dtype, d):
    """Documents of 0 to 3 queries and keys, some rows in front and behind, found among up to 4,099."""
    g = torch.Generator().manual_seed(docs)
    ends = lambda most: torch.cat([torch.tensor([3]), torch.randint(0, most + 1, (docs,), generator=g)]).cumsum(0).to(torch.int32)
    qe, ke = ends(3), ends(2)
    qe[docs // 2:] += 40  # a longer one
    ke[docs // 2:] += 70
    Nq, Nk = int(qe[-1]) + 5, int(ke[-1]) + 2
    H = 2 if docs > 1000 else 4
    q, k, v, dy = make(49 + docs, dtype, 1, H, H // 2, Nq, Nk, d)
    for causal in (False, True):
        check(q, k, v, dy, (docs, causal), causal=causal, q_offsets=qe.cuda(), k_offsets=ke.cuda())


@pytest.mark.parametrize("dtype", [BF, F])
def test_as_many_documents_as_are_taken(dtype):
    """2^20 documents of one token each: their outputs are their values, and nothing but dv has a gradient. Looked through 64 after
    64 they would take minutes."""
    n, d = 1 << 20, 64
    q, k, v, dy = make(50, dtype, 1, 1, 1, n, n, d)
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    o, lse = sv.attention(q, k, v, want_lse=True, q_offsets=off, k_offsets=off)
    assert torch.equal(o, v)
    got = sv.attention_backward(dy, q, k, v, o, lse, q_offsets=off, k_offsets=off)
    # p = 2^(x - lse log2(e)) for lse = x ln(2): two products and two constants, rounded, of the exponent, whose half step is 2^-24 |s|, and two
    # half steps of the exponential: it is no exact 1
    s = (q.double() * k.double()).sum(-1, keepdim=True).abs() * d ** -0.5
    close(got["dv"], dy.double(), 2.0 ** -24 * (2 + 4 * s) * dy.double().abs(), "dv")
    # dy v and dy o differ by the order of their sums
    for name, other in (("dq", k), ("dk", q)):
        bound = 2 * (d + 2) * 2.0 ** -24 * (dy.double().abs() * v.double().abs()).sum(-1, keepdim=True) * other.double().abs() * d ** -0.5
        close(got[name], torch.zeros_like(bound), 2 * bound, name)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("cap", [None, 20.0, 1e4])
def test_scale_of_zero(cap, dtype):
    """All weights are alike, and queries and keys have no gradient."""
    q, k, v, dy = make(51, dtype, 2, 4, 2, 70, 333, 64)
    for kw in ({}, {"causal": True}):
        _, _, got = check(q, k, v, dy, (cap, kw), scale=0.0, cap=cap, **kw)
        assert not got["dq"].any() and not got["dk"].any()
