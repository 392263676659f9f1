"""When a list of gradients gives its device memory back (a stand-in for the
library: no GPU)."""
import gc

import pytest

from paper_2609_36662_gb300 import aloco as A


class _Library:
    """Handles 1, 2, ... and which were destroyed."""

    def __init__(self):
        self.made, self.destroyed = 0, []

    def aloco_grads_create(self, ptrs, sizes, dtypes, n, out):
        self.made += 1
        out._obj.value = self.made
        return A.OK

    def aloco_grads_destroy(self, handle):
        self.destroyed.append(handle.value)

    def aloco_grads_scratch_bytes(self, handle):
        return 64


class _Tensor:
    """As much of a CUDA tensor as a list asks for."""
    is_cuda, device = True, "cuda:0"

    def __init__(self):
        import torch
        self.dtype = torch.float32

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def numel(self):
        return 4

    def _use_count(self):
        return 1

    def is_inference(self):
        return False


@pytest.fixture
def lib(monkeypatch):
    gc.collect()     # lists of other tests
    lib = _Library()
    monkeypatch.setattr(A, "load", lambda: lib)
    monkeypatch.setattr(A, "_lib", lib)
    monkeypatch.setattr(A, "_on_device", lambda device: A._NO_SWITCH)
    if hasattr(A, "_dropped_lists"):
        monkeypatch.setattr(A, "_dropped_lists", [])
    return lib


def test_a_list_that_is_collected_does_not_touch_the_device(lib):
    """Freeing waits for the device, which no stream that is being captured
    allows, and a collection may come at any moment: the memory goes back when the
    next list is made, which waits for the device anyway."""
    a, b = A.GradList([_Tensor()]), A.GradList([_Tensor()])
    a.itself = a                     # a cycle: the collector decides when
    del a
    gc.collect()
    del b
    assert lib.made == 2 and lib.destroyed == []
    c = A.GradList([_Tensor()])
    assert sorted(lib.destroyed) == [1, 2] and lib.made == 3
    del c
    d = A.GradList([_Tensor()])
    assert sorted(lib.destroyed) == [1, 2, 3]
    del d


def test_the_table_of_a_captured_call_is_never_freed(lib, monkeypatch):
    """A graph reads it at every replay, whether or not the list is still there."""
    import torch
    lib.aloco_grad_norm_in = lambda *a: A.OK
    capturing = [False]
    monkeypatch.setattr(A, "_torch", torch)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    cpu = lambda f: lambda *a, **k: f(*a, **{**k, "device": "cpu"})
    monkeypatch.setattr(torch, "zeros", cpu(torch.zeros))
    monkeypatch.setattr(torch, "empty", cpu(torch.empty))
    monkeypatch.setattr(A, "_on_stream", lambda stream, device, inputs: (A._NO_SWITCH, 0))
    lists = []
    for capturing[0] in (False, True):
        lists.append(A.GradList([_Tensor()]))
        A.grad_norm(lists[-1])
    capturing[0] = False
    A.grad_norm(lists[-1])
    del lists[:]
    gc.collect()
    A.GradList([_Tensor()])
    assert lib.destroyed == [1]


def test_a_list_that_was_not_made_leaves_nothing(lib, monkeypatch):
    monkeypatch.setattr(A, "last_error", lambda: "refused")
    lib.aloco_grads_create = lambda *a: A.ERR_ARG
    with pytest.raises(A.AlocoError):
        A.GradList([_Tensor()])
    gc.collect()
    assert lib.destroyed == []
