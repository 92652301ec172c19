"""What the binding refuses, keeps and forgets, on the host alone."""
import copy
import dataclasses
import pickle

import pytest
import torch

from paper_2609_40093_b200 import ep


class _OnDevice:
    """Answers the device query as a tensor of CUDA device 1 would."""
    device = torch.device("cuda", 1)

    def get_device(self):
        return 1


def test_tensors_on_another_device_than_the_current_one_are_refused(monkeypatch):
    """The library launches on the current device: a stream and addresses of another one may not reach it."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    with pytest.raises(ValueError, match="current"):
        ep._stream_of(_OnDevice(), _OnDevice(), None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    assert ep._stream_of(_OnDevice(), _OnDevice(), None) == 0


@pytest.mark.parametrize("kind", ["copy", "deepcopy", "pickle", "asdict"])
def test_a_router_that_was_used_can_be_copied_and_stored(kind):
    """It is a description, kept in configurations and checkpoints; what a call remembers of it is not part of that."""
    router = ep.Router(8, 2, scoring=ep.SCORE_SIGMOID, renormalize=False, scale=2.5, balance_coef=0.1)
    router._struct(torch.zeros(4, 8))
    if kind == "asdict":
        fields = dataclasses.asdict(router)
        assert fields == dict(num_experts=8, top_k=2, scoring=1, renormalize=False, scale=2.5, balance_coef=0.1)
        other = ep.Router(**fields)
    else:
        other = {"copy": copy.copy, "deepcopy": copy.deepcopy, "pickle": lambda r: pickle.loads(pickle.dumps(r))}[kind](router)
    assert other == router and hash(other) == hash(router) and repr(other) == repr(router)
    st, T = other._struct(torch.zeros(5, 8))
    assert T == st.contents.num_tokens == 5 and st.contents.scoring == 1 and router._struct(torch.zeros(4, 8))[0].contents.num_tokens == 4
    assert dataclasses.replace(router, top_k=3)._struct(torch.zeros(4, 8))[0].contents.top_k == 3


@pytest.mark.parametrize("kind", ["copy", "deepcopy", "pickle"])
def test_a_routing_that_was_used_can_be_copied_and_stored(kind, monkeypatch):
    monkeypatch.setattr(ep, "_on_device", lambda *a: None)
    routing = ep.alloc_routing(4, 8, 2, balance=True, device="cpu")
    first = routing._args(4, 8, 2, -1)
    other = {"copy": copy.copy, "deepcopy": copy.deepcopy, "pickle": lambda r: pickle.loads(pickle.dumps(r))}[kind](routing)
    args = other._args(4, 8, 2, -1)
    assert args[0] == other.topk_idx.data_ptr() and args[3] == other.status.data_ptr()
    assert (args[0] == first[0]) == (kind == "copy")
    assert args[2].contents.loss == other.loss.data_ptr()


def test_sizes_past_31_bits_are_refused_not_cut():
    """The library's structs hold 32-bit sizes: 2^32 + 16 tokens would arrive as 16."""
    with pytest.raises(ValueError, match="2\\^31"):
        ep.ep_route(torch.empty(2 ** 32 + 16, 1, device="meta"), ep.Router(1, 1), out=ep.alloc_routing(16, 1, 1, device="cpu"))
    with pytest.raises(ValueError, match="2\\^31"):
        ep.ep_route_workspace_bytes(16, 2, 2 ** 32 + 8)
    x, off = torch.empty(4, 2 ** 32 + 8, dtype=torch.bfloat16, device="meta"), torch.zeros(2, dtype=torch.int32)
    weight = torch.empty(1, 8, 2 ** 32 + 8, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="2\\^31"):
        ep.ep_expert_matmul(x, off, weight, y=torch.empty(4, 8, dtype=torch.bfloat16, device="meta"))
    with pytest.raises(ValueError, match="2\\^31"):
        ep.ep_expert_matmul_backward(torch.empty(4, 8, dtype=torch.bfloat16, device="meta"), x, off, weight)
    with pytest.raises(ValueError, match="2\\^31"):
        ep.alloc_expert_grads(4, 2 ** 32 + 8, 8, 1, device="meta")


def test_a_routing_whose_tensors_changed_in_place_is_checked_again(monkeypatch):
    """The memory may be the same and its extent or order another."""
    monkeypatch.setattr(ep, "_on_device", lambda *a: None)

    def checked():
        r = ep.alloc_routing(4, 8, 4, balance=True, device="cpu")
        r._args(4, 8, 4, -1)
        r._args(4, 8, 4, -1)
        return r

    r = checked()
    at = r.mean_probs.data_ptr()
    r.mean_probs.resize_(4)
    assert r.mean_probs.data_ptr() == at
    with pytest.raises(ValueError, match="mean_probs"):
        r._args(4, 8, 4, -1)
    r = checked()
    r.topk_idx.t_()
    with pytest.raises(ValueError, match="contiguous"):
        r._args(4, 8, 4, -1)
    r = checked()
    r.workspace.resize_(16)
    assert r._args(4, 8, 4, -1)[5] == 16                        # the library refuses it
