"""What the binding of the cache in 8 bits hands to the library: no GPU needed."""
import contextlib
import types

import pytest
import torch

import paper_2606_31315_gb300 as bp
from paper_2606_31315_gb300 import _binding


class OnGpu(torch.Tensor):
    is_cuda = True


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32).as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    calls = []
    for name in ("empty", "zeros"):
        def allocate(*args, _plain=getattr(torch, name), **kwargs):
            kwargs.pop("device", None)
            return _plain(*args, **kwargs).as_subclass(OnGpu)
        monkeypatch.setattr(torch, name, allocate)

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append(a) or 0

    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(_binding, "load", lambda: Lib())
    return calls


@pytest.mark.parametrize("total,room", [((), True), ((0,), True), ((7,), True), ((None,), False)])
def test_pages_update_says_whether_there_is_room_for_new_tokens(calls, total, room):
    """An empty tensor has no address, and a call without any would not look how many new tokens there are."""
    free = i32(9)
    side = types.SimpleNamespace(cuda_stream=0)
    bp.pages_update(i32(2, 4), i32(2), i32(2), free, i32(1), 16, *total, stream=side)
    (a,) = calls
    assert a[9] == (total[0] or 0 if total else 0) and bool(a[10] or a[11]) == room
