"""Checks of the Python entry points that stand between a caller's tensors and the library, without a GPU: the library is
replaced by one that must not be reached, and the checks for a GPU are left out."""
import pytest
import torch

import paper_2603_08982_amd as sv
from paper_2603_08982_amd import binding


class Reached(Exception):
    pass


class NoLibrary:
    def __getattr__(self, name):
        def call(*args):
            raise Reached(name)

        return call


@pytest.fixture
def no_library(monkeypatch):
    monkeypatch.setattr(binding, "load_library", NoLibrary)
    monkeypatch.setattr(binding, "_need_gpu", lambda *ts: None)
    monkeypatch.setattr(binding, "_stream", lambda: 0)


OP = (1, 2, 24, 64)
BAD_OUT = {
    "fewer tokens": lambda: torch.empty(1, 2, 23, 64),
    "fewer heads": lambda: torch.empty(1, 1, 24, 64),
    "a smaller type": lambda: torch.empty(*OP, dtype=torch.bfloat16),
    "another device": lambda: torch.empty(*OP, device="meta"),
    "d not contiguous": lambda: torch.empty(1, 2, 64, 24).transpose(2, 3),
}


@pytest.mark.parametrize("what", BAD_OUT)
def test_unpermute_refuses_an_output_that_is_not_its_own(no_library, what):
    op, perm = torch.zeros(*OP), torch.zeros(1, 2, 24, dtype=torch.int32)
    with pytest.raises(sv.SvgearError):
        sv.unpermute(op, perm, BAD_OUT[what]())
    with pytest.raises(Reached):
        sv.unpermute(op, perm, torch.empty(1, 24, 2, 64).transpose(1, 2))


@pytest.mark.parametrize("perm", [(1, 2, 23), (1, 1, 24), (2, 24)], ids=str)
def test_unpermute_refuses_a_permutation_of_other_tokens(no_library, perm):
    op = torch.zeros(*OP)
    with pytest.raises(sv.SvgearError):
        sv.unpermute(op, torch.zeros(*perm, dtype=torch.int32))
    with pytest.raises(sv.SvgearError):
        sv.unpermute(op, torch.zeros(1, 2, 24, dtype=torch.int64))


@pytest.mark.parametrize("token_order", [False, True])
@pytest.mark.parametrize("what", BAD_OUT)
def test_layer_refuses_such_an_output_before_its_centroids_change(no_library, what, token_order):
    q = torch.zeros(*OP)
    c = torch.zeros(1, 2, 3, 64)
    with pytest.raises(sv.SvgearError):
        sv.attention_layer(q, q, q, c, c.clone(), 1, 100, overlap=False, token_order=token_order, out=BAD_OUT[what]())
    with pytest.raises(Reached, match="kmeans"):
        sv.attention_layer(q, q, q, c, c.clone(), 1, 100, overlap=False, token_order=token_order, out=torch.empty(*OP))


@pytest.fixture
def no_device(no_library, monkeypatch):
    """The same for the entry points that take strides, whose tensors are then on no device at all (they have sizes alone)."""
    import contextlib

    monkeypatch.setattr(binding, "_on_device", lambda device: contextlib.nullcontext())
    monkeypatch.setattr(binding, "_stream_of", lambda device: 0)


def meta(*shape, strides=None, dtype=torch.bfloat16):
    t = torch.empty(1, dtype=dtype, device="meta")
    if strides is None:
        return torch.empty(*shape, dtype=dtype, device="meta")
    return t.expand(*shape) if strides == "one" else t.as_strided(shape, strides)


# sizes whose low 32 bits are an ordinary call's, and the first past each limit
PAST = 1 << 32
TOO_LARGE = {
    "batch entries past 32 bits": lambda: sv.linear(meta(1, 1, 8).expand(PAST + 1, 1, 8), meta(16, 8)),
    "d_in past 32 bits": lambda: sv.linear(meta(1, 2, PAST + 8), meta(16, PAST + 8)),
    "d_out past 32 bits": lambda: sv.linear(meta(1, 2, 8), meta(PAST + 16, 8)),
    "rows past 2^30": lambda: sv.linear(meta(1, 1, 8).expand(1 << 15, (1 << 15) + 1, 8), meta(16, 8)),
    "d_in past 2^21": lambda: sv.linear(meta(1, 2, (1 << 21) + 1), meta(16, (1 << 21) + 1)),
    "backward, batch entries past 32 bits": lambda: sv.linear_backward(meta(1, 1, 16).expand(PAST + 1, 1, 16), None, meta(16, 8), want=["dx"]),
    "backward, d_in past 32 bits": lambda: sv.linear_backward(meta(1, 2, 16), None, meta(16, PAST + 8), want=["dx"]),
    "backward, d_out past 32 bits": lambda: sv.linear_backward(meta(1, 2, PAST + 16), meta(1, 2, 8), None, want=["dw"]),
    "backward, dbias alone": lambda: sv.linear_backward(meta(1, 2, PAST + 16), None, None, want=["dbias"]),
}


@pytest.mark.parametrize("what", TOO_LARGE)
def test_linear_refuses_sizes_that_its_arguments_do_not_hold(no_device, what):
    with pytest.raises(sv.SvgearError):
        TOO_LARGE[what]()


def test_linear_of_the_largest_sizes_goes_on(no_device):
    with pytest.raises(Reached):
        sv.linear(meta(1, 1, 1 << 21).expand(1 << 15, 1 << 15, 1 << 21), meta(1 << 21, 1 << 21))
    with pytest.raises(Reached):
        sv.linear_backward(meta(1, 1, 1 << 21).expand(1 << 15, 1 << 15, 1 << 21), None, meta(1 << 21, 1 << 21), want=["dx"])


def rotary_call(back, shape=(1, 2, 24, 64), sections=(10, 11, 11), **kw):
    q = meta(1, 1, 1, shape[3]).expand(*shape)
    f = torch.empty(sum(sections), dtype=torch.float64, device="meta")
    if "positions" not in kw:
        kw.setdefault("grid", (2, 3, 4))
    return sv.rotary_backward([q], None, f, sections, **kw) if back else sv.rotary([q], f, sections, **kw)


ROTARY_TOO_LARGE = {
    "batch entries": dict(shape=(PAST + 1, 2, 24, 64)),
    "heads": dict(shape=(1, PAST + 2, 24, 64)),
    "tokens": dict(shape=(1, 1, (1 << 30) + 1, 64), grid=((1 << 30) + 1, 1, 1)),
    "elements of a head": dict(shape=(1, 2, 24, PAST + 64)),
    "text tokens": dict(n_tail=(1 << 64) + 1),
    "text tokens below none": dict(n_tail=-(1 << 64) + 1),
    "first": dict(first=1 << 64),
    "first below none": dict(first=-(1 << 64)),
    "grid": dict(grid=((1 << 64) + 2, 3, 4)),
    "grid past 31 bits": dict(grid=(1 << 31, 1, 1)),
    "sections": dict(sections=(PAST + 10, 11 - PAST, 11)),
}


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("what", ROTARY_TOO_LARGE)
def test_rotary_refuses_sizes_that_its_arguments_do_not_hold(no_device, what, back):
    with pytest.raises(sv.SvgearError):
        rotary_call(back, **ROTARY_TOO_LARGE[what])


@pytest.mark.parametrize("back", [False, True])
def test_rotary_of_the_largest_sizes_goes_on(no_device, back):
    for kw in (dict(), dict(shape=(1, 128, 1 << 23, 128), grid=(1 << 30, 1, 1), first=(1 << 30) - (1 << 23)),
               dict(shape=(1 << 15, 1, 1 << 15, 64), grid=(1 << 15, 1, 1)), dict(n_tail=23, grid=((1 << 31) - 1, 1, 1)),
               dict(positions=torch.empty(24, 3, dtype=torch.int32, device="meta"), first=1 << 64)):
        with pytest.raises(Reached):
            rotary_call(back, **kw)


def test_block_runs_on_its_tensors_device(monkeypatch):
    """Every call of the block, the layer's too, is made with x's device as the current one."""
    import contextlib

    seen, current = [], []

    @contextlib.contextmanager
    def on(device):
        current.append(device)
        yield
        current.pop()

    def linear(x, w, *a, **kw):
        seen.append(("linear", tuple(current)))
        return x.new_empty(*x.shape[:-1], w.shape[0]), None

    def layer(q, k, v, *a, **kw):
        seen.append(("attention_layer", tuple(current)))
        return None, {}

    monkeypatch.setattr(binding, "_need_gpu", lambda *ts: None)
    monkeypatch.setattr(binding, "_on_device", on)
    monkeypatch.setattr(binding, "linear", linear)
    monkeypatch.setattr(binding, "rotary", lambda *a, **kw: seen.append(("rotary", tuple(current))))
    monkeypatch.setattr(binding, "attention_layer", layer)
    x, c = meta(1, 24, 32), meta(1, 2, 3, 64, dtype=torch.float32)
    y, _ = sv.attention_block(x, meta(3 * 128, 32), meta(40, 128), c, c, 1, 100, meta(32, dtype=torch.float64), (10, 11, 11), grid=(2, 3, 4))
    assert y.shape == (1, 24, 40)
    assert seen == [(name, (x.device,)) for name in ("linear", "rotary", "attention_layer", "linear")]
    assert not current


def test_block_refuses_centroids_of_another_device(no_device):
    x, c = meta(1, 24, 32), meta(1, 2, 3, 64, dtype=torch.float32)
    for q, k in ((torch.zeros(1, 2, 3, 64), c), (c, torch.zeros(1, 2, 3, 64))):
        with pytest.raises(sv.SvgearError):
            sv.attention_block(x, meta(3 * 128, 32), meta(40, 128), q, k, 1, 100, meta(32, dtype=torch.float64), (10, 11, 11), grid=(2, 3, 4))


BAD_CENTROIDS = [(2, 2, 3, 64), (1, 1, 3, 64), (1, 2, 3, 128), (2, 3, 64)]


@pytest.mark.parametrize("shape", BAD_CENTROIDS, ids=str)
def test_kmeans_refuses_centroids_of_other_heads(no_library, shape):
    """They are written, [B,H,C,d] of them."""
    x = torch.zeros(*OP)
    with pytest.raises(sv.SvgearError):
        sv.kmeans(x, torch.zeros(*shape), 1)
    with pytest.raises(Reached):
        sv.kmeans(x, torch.zeros(1, 2, 3, 64), 1)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("shape", BAD_CENTROIDS, ids=str)
def test_layer_and_block_refuse_centroids_of_other_heads(no_device, shape, which):
    """Before anything is launched: the queries' k-means would have changed its centroids."""
    q, good, bad = torch.zeros(*OP), torch.zeros(1, 2, 3, 64), torch.zeros(*shape)
    init = (bad, good) if which == 0 else (good, bad)
    with pytest.raises(sv.SvgearError):
        sv.attention_layer(q, q, q, *init, 1, 100, overlap=False)
    x, w, o, f = torch.zeros(1, 24, 32), torch.zeros(3 * 128, 32), torch.zeros(40, 128), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(sv.SvgearError):
        sv.attention_block(x, w, o, *init, 1, 100, f, (10, 11, 11), grid=(2, 3, 4))
