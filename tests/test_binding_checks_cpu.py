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
