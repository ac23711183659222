"""A workspace of the gradient norm on another device than the current one is refused before the library is called, as that
of every other operator.  The devices are made up; no GPU needed."""
import array

import pytest
import torch

from paper_2605_09825_b200 import api


class Workspace:
    is_cuda = True

    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return 1 << 20


class Library:
    calls = 0

    def mxfp4_grad_norm_workspace_bytes(self, count):
        return 4736

    def mxfp4_grad_norm(self, *args):
        self.calls += 1
        return 0

    mxfp4_clip_grads = mxfp4_grad_norm


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    empty = torch.empty
    monkeypatch.setattr(api, "load_library", lambda: lib)
    monkeypatch.setattr(api, "_tensor_list", lambda tensors, name: (array.array("q", [4096]), array.array("q", [8]), array.array("i", [0])))
    monkeypatch.setattr(api, "_raw_stream", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch, "empty", lambda *s, device=None, **kw: empty(*s, **kw))
    return lib


CALLS = {"norm": lambda ws: api.grad_norm([torch.zeros(8)], ws), "clip": lambda ws: api.clip_grads([torch.zeros(8)], 1.0, workspace=ws)}


@pytest.mark.parametrize("name", CALLS)
def test_a_workspace_on_another_device_is_refused(library, name):
    with pytest.raises(ValueError):
        CALLS[name](Workspace(1))
    assert library.calls == 0


@pytest.mark.parametrize("name", CALLS)
def test_one_on_the_current_device_and_none_are_taken(library, name):
    CALLS[name](Workspace(0))
    CALLS[name](None)
    assert library.calls == 2
